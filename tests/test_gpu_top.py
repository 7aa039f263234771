"""Top alternatives, log-probs and entropy of given logits against 64 bits, where they can go wrong.

Bounds.  U = 2^-24 is half a step of fp32; s = z / T.  The scale log2(e) / T is rounded once, which moves every s by U |s|, and the exponents u = (z - m) scale are
rounded to U |u|; where u = 0 is taken to, m scale, cancels.  A thread adds one 512th of the row's exponentials, in sums of 16 to a tile, the lanes, waves and
parts another 30 at most (a row of up to 65536 logits may go to 128 threads, four times as many to each: the bound below is held there without that
factor), each exponential is good to 2 U: lse is off by A = (V / 512 + 16 + 40) U + 4 U max |s|, and log-probs by that and the rounding of the result.  The entropy takes a second such sum, of 2^u u, whose size is the entropy's and a little, and changes by the variance of s
(at most a quarter of its squared range) times what s is off by relative to itself."""
import numpy as np
import pytest
import torch

from tests import top_oracle as to
from tests.top_oracle import f64, rand

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def mrl():
    import paper_2605_07244_amd as m
    m.lib()
    return m


def _near(name, got, want, bound):
    got, want = f64(got), np.asarray(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), name
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), name
    ok = np.isfinite(want)
    err, bound = np.abs(got - np.where(ok, want, got)), np.broadcast_to(bound, want.shape)
    worst = float(np.max(err[ok] / bound[ok])) if ok.any() else 0.0
    print(f"{name}: worst error over its bound {worst:.3f}")
    assert worst <= 1.0, (name, worst)


def _check(mrl, z, k, targets=None, mask=None, T=1.0, **kw):
    r = mrl.top_logprobs(z, k, target_ids=targets, token_mask=mask, temperature=T, **kw)
    torch.cuda.synchronize()
    z64 = f64(z)
    N, V = z64.shape
    ids, top, lse, entropy, logp = to.top(z64, k, T)
    on = np.ones(N, dtype=bool) if mask is None else mask.cpu().numpy() != 0
    with np.errstate(all="ignore"):
        s = np.where(np.isfinite(z64), z64 / T, np.nan)
        most = np.nan_to_num(np.nanmax(np.abs(s), 1)) if V else np.zeros(N)
        spread = np.nan_to_num(np.nanmax(s, 1) - np.nanmin(s, 1))
    spread = np.minimum(spread, 200.0)                  # (what is further below has no probability)
    A = (V / 512 + 16 + 40) * U + 4 * U * most
    if k:
        assert np.array_equal(r["ids"].cpu().numpy(), np.where(on[:, None], ids, -1))
        _near("top", r["top_logp"], np.where(on[:, None], top, 0.0), A[:, None] + 2 * U * np.abs(np.nan_to_num(top, neginf=0)) + 1e-30)
    else:
        assert r["ids"] is None and r["top_logp"] is None
    _near("lse", r["lse"], np.where(on, lse, 0.0), A + U * np.nan_to_num(np.abs(lse)) + 1e-30)
    _near("entropy", r["entropy"], np.where(on, entropy, 0.0), (2 + np.nan_to_num(entropy)) * A + U * spread ** 2 / 4 + 1e-30)
    if targets is not None:
        y = targets.cpu().numpy()
        ok = on & (y >= 0) & (y < V)
        want = np.where(ok, logp[np.arange(N), np.clip(y, 0, V - 1)], 0.0)
        _near("logp", r["logp"], want, A + 2 * U * np.abs(np.nan_to_num(want, neginf=0)) + 1e-30)
    return r


@pytest.mark.parametrize("N,V,k", [(1, 1, 1), (1, 2, 2), (3, 7, 7), (2, 63, 5), (5, 64, 64), (4, 129, 100), (1, 513, 256), (1, 4096, 256), (1, 8191, 1), (2, 8192, 200), (3, 8193, 33),
                                   (1, 50257, 50), (40, 12345, 256), (700, 300, 3), (1030, 9000, 64), (600, 20011, 256), (17, 151936, 20)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_sizes(mrl, N, V, k, dtype):
    z = rand((N, V), dtype, N + V + k, 3.0)
    targets = torch.randint(-1, V + 1, (N,), device="cuda", dtype=torch.int32, generator=torch.Generator("cuda").manual_seed(V))
    _check(mrl, z, k, targets, T=1.0 if V % 2 else 0.7)


@pytest.mark.parametrize("T", [0.1, 0.5, 2.0, 30.0])
def test_temperatures(mrl, T):
    _check(mrl, rand((6, 5003), F32, 3, 2.0), 17, torch.arange(6, device="cuda", dtype=torch.int32), T=T)


@pytest.mark.parametrize("N", [2, 1100])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_that_defeat_the_bound(mrl, N, dtype):
    """Sorted both ways, constant, few values, all large ones in one thread's elements: the list overflows or is all ties."""
    V = 20000
    up = torch.arange(V, device="cuda", dtype=F32) / 1000 - 10
    few = (torch.arange(V, device="cuda") % 3).float()
    one = torch.where(torch.arange(V, device="cuda") % 4096 < 8, 5.0, 0.0) + up / 100
    rows = torch.stack([up, up.flip(0), torch.full_like(up, 1.5), few, one, torch.full_like(up, -3.0)])
    z = rows[torch.arange(N, device="cuda") % 6].to(dtype).contiguous()
    for k in (1, 40, 256):
        _check(mrl, z[:6] if N > 6 else z, k)
        r = mrl.top_logprobs(z, k)
        assert torch.equal(r["ids"][:6], mrl.top_logprobs(z[:6].contiguous(), k)["ids"])
        assert torch.equal(r["ids"], r["ids"][:6][torch.arange(N, device="cuda") % 6])


@pytest.mark.parametrize("V", [9, 700, 30011])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_infinities_nan_and_lowest_values(mrl, V, dtype):
    inf, low = float("inf"), torch.finfo(dtype).min
    z = rand((14, V), dtype, V, 2.0)
    z[0, 3] = float("nan")
    z[1, V - 1] = inf
    z[2] = -inf
    z[3] = -inf
    z[3, V // 2] = 0.5                                  # one token left
    z[4, ::2] = -inf
    z[5] = low
    z[6] = low
    z[6, 5] = 2.0
    z[7, 1:] = low
    z[8, 0], z[8, 1] = inf, float("nan")
    z[9] = -inf
    z[9, 1] = float("nan")
    z[10, :4] = torch.tensor([0.0, -0.0, 0.0, -0.0], device="cuda")
    z[10, 4:] = -1.0
    z[11] = torch.finfo(dtype).max
    z[12] = -1e30
    z[13, 2] = low
    for k in (0, 1, 9):
        _check(mrl, z, k, torch.full((14,), 5, device="cuda", dtype=torch.int32))
    many = z.repeat(80, 1)
    for k in (0, 9):
        a, b = mrl.top_logprobs(many, k), mrl.top_logprobs(z, k)      # a workgroup a row, and several
        if k:
            assert torch.equal(a["ids"].view(80, 14, k), b["ids"].expand(80, 14, k))
        assert torch.equal(torch.isnan(a["lse"]).view(80, 14), torch.isnan(b["lse"]).expand(80, 14))
        assert torch.allclose(a["lse"].view(80, 14), b["lse"].expand(80, 14), rtol=1e-6, atol=1e-5, equal_nan=True)


@pytest.mark.parametrize("N", [2, 1100])
@pytest.mark.parametrize("V", [9, 700, 30011])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [1.0, 0.7])
def test_log_probs_of_logits_far_from_zero(mrl, N, V, dtype, T):
    """Rows masked throughout with the type's lowest value, and others whose logits have much in common: log-probs are those of the differences."""
    low = torch.finfo(dtype).min
    far = [low, low / 2, -1e30, -1e20, -1e9, 1e5, 1e9, 3e9, 1e15, 1e30, 1e36]
    z = torch.tensor(far, device="cuda").to(dtype)[:, None].repeat(1, V)
    z[5:8, 1::3] -= z[5:8, 1::3].abs() * 2.0 ** -7      # (3e9 too: by 2e7)
    z[0, 4], z[4, 4] = low / 2, 0.0                 # one that is not masked
    target = torch.tensor([0, 4] * 6, device="cuda", dtype=torch.int32)[:len(far)]
    x = z.double().cpu().numpy()
    s = (x - x.max(1, keepdims=True)) / T
    want = s - np.log(np.exp(s).sum(1, keepdims=True))
    k = min(V, 7)
    ids = to.top(x, k)[0]
    p = np.exp(want)
    entropy = -(p * np.where(p > 0, want, 0.0)).sum(1)
    many = z.repeat(-(-N // len(far)), 1)
    r = mrl.top_logprobs(many, k, target_ids=target.repeat(len(many) // len(far)), temperature=T)
    # The exponents' residue where the largest logit is taken to is 128 at most (beyond that the row is summed anew), rounded to U of itself; the scale is rounded by U, which
    # moves differences; sums as above; then the results' rounding.
    A = (V / 512 + 16 + 40) * U + 4 * U * 128
    for n in range(0, len(many), len(far)):
        rows = slice(n, n + len(far))
        assert np.array_equal(r["ids"][rows].cpu().numpy(), ids)
        for name, got, exact in (("top", r["top_logp"], np.take_along_axis(want, ids, 1)), ("logp", r["logp"], want[np.arange(len(far)), target.cpu().numpy()])):
            with np.errstate(over="ignore"):
                exact = exact.astype(np.float32).astype(np.float64)      # (the lowest value over 0.7 is no float)
            _near(name, got[rows], exact, A + 4 * U * np.abs(np.where(np.isfinite(exact), exact, 0.0)))
        _near("entropy", r["entropy"][rows], entropy, (2 + entropy) * A + 4 * U * 200)
        if n == 0 and V == 9:
            assert abs(float(r["top_logp"][2, 0]) + np.log(9.0)) <= A + U * 3


@pytest.mark.parametrize("V", [9, 700, 30011])
@pytest.mark.parametrize("N", [2, 1100])
def test_logits_that_fill_the_range(mrl, N, V):
    # At this temperature the scale is 8192, a power of two, so that the largest float over it, scaled, is the largest float exactly: its distance from where
    # a thread's running maximum begins is infinite, though the sum of exponentials is not.  Three such logits: entropy log 3, good to the rounding of the result.
    T = float(np.float32(1.4426950408889634 / 8192))
    assert np.float32(1.4426950408889634 / T) == np.float32(8192)
    z = torch.zeros((N, V), device="cuda")
    z[:, [1, 4, 8]] = torch.finfo(F32).max / 8192
    r = mrl.top_logprobs(z, 3, temperature=T)
    assert torch.equal(r["ids"], torch.tensor([1, 4, 8], dtype=torch.int32, device="cuda").expand(N, 3))
    _near("entropy", r["entropy"], np.full(N, np.log(3.0)), 4 * U * np.log(3.0))
    want = float(z[0, 1]) / T
    _near("lse", r["lse"], np.full(N, want), 4 * U * want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V,pad,first", [(1000, 1, 0), (1001, 7, 3), (50000, 13, 5)])
def test_rows_that_begin_anywhere(mrl, dtype, V, pad, first):
    wide = rand((9, V + pad + first), dtype, V, 2.0)
    wide[:, V + first:] = float("nan")                 # (never read)
    wide[:, :first] = float("inf")
    z = wide[:, first:first + V]
    a = _check(mrl, z, 25, torch.arange(9, device="cuda", dtype=torch.int32))
    b = mrl.top_logprobs(z.contiguous(), 25)
    assert torch.equal(a["ids"], b["ids"]) and torch.equal(a["top_logp"], b["top_logp"]) and torch.equal(a["entropy"], b["entropy"])


@pytest.mark.parametrize("N", [5, 1500])
def test_masked_rows_are_not_read(mrl, N):
    z = rand((N, 3001), F32, 8, 2.0)
    mask = (torch.arange(N, device="cuda") % 3 != 1).to(torch.uint8)
    z[mask == 0] = float("nan")
    _check(mrl, z, 11, torch.zeros(N, device="cuda", dtype=torch.int32), mask)
    r = mrl.top_logprobs(z, 11, token_mask=torch.zeros_like(mask))
    assert torch.all(r["ids"] == -1) and torch.all(r["top_logp"] == 0) and torch.all(r["lse"] == 0) and r["logp"] is None


@pytest.mark.parametrize("N,V,k,dtype", [(1030, 300001, 64, BF16), (1030, 300001, 256, F32), (2, 1 << 24, 100, F32), (3, 5000011, 7, BF16), (1030, 65536, 32, F32), (1030, 32768, 64, BF16)])
def test_long_rows(mrl, N, V, k, dtype):
    """Rows of more tiles than a workgroup has notes for, whole and in slices; the reference in 64 bits on the GPU."""
    z = rand((N, V), dtype, N, 3.0)
    z[0, V - 1] = 40.0
    r = mrl.top_logprobs(z, k)
    for n in (0, 1, N - 1):
        x = z[n].double()
        order = torch.sort(x, descending=True, stable=True).indices[:k]
        assert torch.equal(r["ids"][n].long(), order)
        lse = torch.logsumexp(x, 0)
        p = torch.exp(x - lse)
        A = (V / 512 + 56) * U + 4 * U * float(x.abs().max())
        assert abs(float(r["lse"][n]) - float(lse)) <= A + U * float(lse)
        assert float((r["top_logp"][n].double() - (x[order] - lse)).abs().max()) <= A + 40 * U
        H = float(lse - (p * x).sum())
        assert abs(float(r["entropy"][n]) - H) <= (2 + H) * A + U * 200 ** 2 / 4


@pytest.mark.parametrize("N,V,k", [(1, 65537, 8), (31, 65537, 20), (1, 151553, 13), (1, 63489, 2), (1, 151557, 13)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_last_slice_shorter_than_the_list(mrl, N, V, k, dtype):
    """Rows in slices of which the last has one logit, or five: what calls with larger logits left in the chip's memory is none of theirs."""
    mrl.top_logprobs(rand((2048, 70001), dtype, 1, 3.0) + 5000.0, 256)      # (a workgroup a row: their lists)
    z = rand((N, V), dtype, N + V + k, 3.0)
    _check(mrl, z, k, T=0.7)
    z[:, V - 1] = 50.0                                  # and the last logit counts
    _check(mrl, z, k)


@pytest.mark.parametrize("N", [3, 1100])
def test_one_thread_holds_the_largest(mrl, N):
    """All alternatives among the logits that one thread of the workgroup looks at; and more equal logits than the list holds."""
    V = 60000
    z = torch.zeros((N, V), device="cuda")
    z[:, 4096 * torch.arange(14, device="cuda")] = torch.arange(14, device="cuda").float() + 1
    z[:, 30000:] -= 1.0
    z[:, 100:5000] = 0.25
    _check(mrl, z[:3].contiguous(), 30)
    r = mrl.top_logprobs(z, 30)
    assert torch.equal(r["ids"], mrl.top_logprobs(z[:3].contiguous(), 30)["ids"][:1].expand(N, 30))


def test_no_rows_and_outputs_left_out(mrl):
    r = mrl.top_logprobs(torch.empty(0, 100, device="cuda"), 5)
    assert r["ids"].shape == (0, 5) and r["lse"].shape == (0,)
    z = rand((3, 100), F32, 1)
    a, b = mrl.top_logprobs(z, 5), mrl.top_logprobs(z, 5, want_lse=False, want_entropy=False)
    assert b["lse"] is None and b["entropy"] is None and torch.equal(a["top_logp"], b["top_logp"])
    c = mrl.top_logprobs(z, 0, want_entropy=False)
    assert torch.equal(a["lse"], c["lse"])


def test_offsets_beyond_32_bits(mrl):
    N, V = 14400, 151936                               # 4.4 GB, 2.19e9 elements
    z = torch.zeros((N, V), device="cuda", dtype=BF16)
    for n in (0, 14133, N - 1):
        z[n] = rand((V,), BF16, n, 3.0)
    r = mrl.top_logprobs(z, 30)
    for n in (0, 14133, N - 1):
        ids, top, lse, _, _ = to.top(f64(z[n:n + 1]), 30)
        assert np.array_equal(r["ids"][n:n + 1].cpu().numpy(), ids) and abs(float(r["lse"][n]) - lse[0]) < 1e-4


def test_captured_calls_share_a_workspace_in_order(mrl):
    z = rand((4, 30000), F32, 5, 3.0)
    want = mrl.top_logprobs(z, 20)
    ws = torch.empty(mrl.lib().mrl_top_logprobs_workspace(4, 30000, 20), dtype=torch.uint8, device="cuda")
    other = rand((4, 30000), F32, 6, 3.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            a = mrl.top_logprobs(z, 20, workspace=ws)
            b = mrl.top_logprobs(other, 20, workspace=ws)
    want_b = mrl.top_logprobs(other, 20)
    for _ in range(4):
        for t in (a["ids"], b["ids"], a["top_logp"], a["entropy"]):
            t.zero_()
        ws.random_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a["ids"], want["ids"]) and torch.equal(a["top_logp"], want["top_logp"]) and torch.equal(a["entropy"], want["entropy"])
        assert torch.equal(b["ids"], want_b["ids"])
    z.copy_(other)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a["ids"], want_b["ids"]) and torch.equal(a["entropy"], want_b["entropy"])


def test_two_streams(mrl):
    z = [rand((3, 100000), F32, i, 3.0) for i in range(2)]
    want = [mrl.top_logprobs(x, 50) for x in z]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s, x in zip(streams, z):
        with torch.cuda.stream(s):
            got.append([mrl.top_logprobs(x, 50) for _ in range(5)])
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        for r in g:
            assert all(torch.equal(r[n], w[n]) for n in ("ids", "top_logp", "lse", "entropy"))
