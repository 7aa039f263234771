"""Embedding lookup and its gradient against 64 bits, where they can go wrong.

Bounds.  U = 2^-24 is half a step of fp32, HALF that of an output's type.  The lookup rounds scale (once, to fp32), the product and the output.  A gradient of m rows adds
them one after the other, in groups whose sums are added likewise: at most m roundings of partial sums no larger than the sum of magnitudes, the scale's and the
product's roundings, one of an old value's sum, and the output's."""
import numpy as np
import pytest
import torch

from tests import top_oracle as to
from tests.top_oracle import f64, rand

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: U, BF16: 2.0 ** -8}


@pytest.fixture(scope="module")
def mrl():
    import paper_2605_07244_amd as m
    m.lib()
    return m


def _ids(N, V, seed, low=0, high=None):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randint(low, V if high is None else high, (N,), device="cuda", generator=g, dtype=torch.int32)


@pytest.mark.parametrize("d", [1, 2, 7, 8, 9, 15, 63, 64, 100, 511, 713, 2048, 4100])
@pytest.mark.parametrize("table,out", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)])
def test_lookup(mrl, d, table, out):
    N, V = 1003, 77
    t = rand((V, d), table, d)
    ids = _ids(N, V, d, -2, V + 2)
    mask = (torch.arange(N, device="cuda") % 5 != 2).to(torch.uint8)
    for scale, m in ((1.0, None), (d ** 0.5, mask), (-0.3, None)):
        y = mrl.embedding(t, ids, scale, m, out)
        i = ids.cpu().numpy()
        on = (i >= 0) & (i < V) & (True if m is None else m.cpu().numpy() != 0)
        want = np.where(on[:, None], f64(t)[np.clip(i, 0, V - 1)] * scale, 0.0)
        assert y.shape == (N, d) and y.dtype == out
        assert np.all(np.abs(f64(y) - want) <= (3 * U + HALF[out]) * np.abs(want))
        assert np.all(f64(y)[~on] == 0)


@pytest.mark.parametrize("N", [1, 2, 3, 255, 4097])
def test_lookup_of_few_and_many(mrl, N):
    t = rand((50, 520), BF16, N)
    ids = _ids(N, 50, N)
    assert torch.equal(mrl.embedding(t, ids), t[ids.long()])
    out = torch.full((N, 520), 7.0, device="cuda", dtype=BF16)
    assert mrl.embedding(t, ids, out=out) is out and torch.equal(out, t[ids.long()])


def test_lookup_none(mrl):
    t = rand((5, 12), F32, 0)
    t[0] = float("nan")                                # (what no token names is not seen)
    y = mrl.embedding(t, torch.full((9,), -1, device="cuda", dtype=torch.int32))
    assert torch.all(y == 0)
    assert mrl.embedding(t, torch.empty(0, device="cuda", dtype=torch.int32)).shape == (0, 12)


def test_lookup_behind_32_bits(mrl):
    t = torch.empty((530000, 4100), device="cuda", dtype=BF16)           # 2.17e9 elements
    t[529999] = rand((4100,), BF16, 1)
    t[3] = rand((4100,), BF16, 2)
    ids = torch.tensor([529999, 3, 529999], device="cuda", dtype=torch.int32)
    assert torch.equal(mrl.embedding(t, ids), t[ids.long()])
    n = 530001
    many = torch.full((n,), 3, device="cuda", dtype=torch.int32)
    many[-1] = 529999
    y = mrl.embedding(t, many)
    assert torch.equal(y[-1], t[529999]) and torch.equal(y[-2], t[3]) and torch.equal(y[0], t[3])


def _check_back(mrl, dy, ids, V, scale=1.0, mask=None, out=F32, base=None):
    got = mrl.embedding_backward(dy, ids, V, scale, mask, out_dtype=out if base is None else None, out=None if base is None else base.clone(), accumulate=base is not None)
    want, mag, count = to.embedding_backward(f64(dy), ids.cpu().numpy(), V, scale, None if mask is None else mask.cpu().numpy())
    old = np.zeros_like(want) if base is None else f64(base)
    err = np.abs(f64(got) - want - old)
    bound = (count[:, None] + 3) * U * mag + HALF[got.dtype] * np.abs(want + old) + (U * np.abs(old) if base is not None else 0.0)
    assert got.shape == (V, dy.shape[1]) and np.all(np.isfinite(err))
    assert np.all(err <= bound), float(np.max(err / np.maximum(bound, 1e-300)))
    if base is None:
        assert np.all(f64(got)[count == 0] == 0)
    else:
        untouched = torch.from_numpy(count == 0).cuda()
        assert torch.equal(got[untouched], base[untouched])
    return got


@pytest.mark.parametrize("N", [1, 2, 7, 8, 9, 15, 16, 17, 33, 64, 65, 1000, 4095, 4096, 4097, 8193, 20000])
@pytest.mark.parametrize("V", [1, 3, 511, 512, 5000])
def test_gradient_sizes(mrl, N, V):
    _check_back(mrl, rand((N, 72), F32, N + V), _ids(N, V, N * V, -1, V + 1), V, 1.7)


@pytest.mark.parametrize("N", [100, 10000])
@pytest.mark.parametrize("V", [262143, 262144, 300001])
def test_gradient_of_many_ids(mrl, N, V):
    """Two passes and three; ids at both ends of the table."""
    ids = _ids(N, V, N)
    ids[::7] = V - 1
    ids[::11] = 0
    _check_back(mrl, rand((N, 16), BF16, N), ids, V)


@pytest.mark.parametrize("d", [1, 3, 7, 8, 9, 100, 511, 512, 513, 713, 1536, 2050, 4104])
@pytest.mark.parametrize("dy,out", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
def test_gradient_widths(mrl, d, dy, out):
    N, V = 700, 60
    mask = (torch.arange(N, device="cuda") % 4 != 3).to(torch.uint8)
    x = rand((N, d), dy, d)
    x[mask == 0] = float("nan")                        # (never read)
    _check_back(mrl, x, _ids(N, V, d), V, d ** 0.5, mask, out)


@pytest.mark.parametrize("N", [50, 5000, 70000])
def test_one_token_all_over(mrl, N):
    """A single token's rows reach over all chunks; a few others between them."""
    ids = torch.full((N,), 5, device="cuda", dtype=torch.int32)
    ids[N // 2] = 2
    ids[N // 3] = 9
    _check_back(mrl, rand((N, 40), F32, N), ids, 11)
    _check_back(mrl, rand((N, 40), BF16, N), torch.full_like(ids, 10), 11)


def test_common_tokens(mrl):
    N, V = 30000, 9000
    u = torch.rand(N, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    ids = (torch.exp(u * np.log(V)) - 1).int().clamp_(0, V - 1)
    _check_back(mrl, rand((N, 1024), BF16, 1), ids, V)


@pytest.mark.parametrize("N,d", [(300, 520), (9000, 136)])
def test_accumulation_into_a_shared_head(mrl, N, d):
    V = 700
    _check_back(mrl, rand((N, d), BF16, N), _ids(N, V, N), V, 0.5, base=rand((V, d), F32, N + 1))


def test_no_tokens(mrl):
    none = torch.empty(0, device="cuda", dtype=torch.int32)
    dy = torch.empty((0, 20), device="cuda")
    out = torch.full((7, 20), 3.0, device="cuda")
    assert torch.all(mrl.embedding_backward(dy, none, 7) == 0)
    assert torch.all(mrl.embedding_backward(dy, none, 7, out=out, accumulate=True) == 3)
    assert torch.all(mrl.embedding_backward(dy, none, 7, out=out) == 0) and torch.all(out == 0)
    for bad in (-1, 7):
        assert torch.all(mrl.embedding_backward(torch.full((30, 20), float("nan"), device="cuda"), torch.full((30,), bad, device="cuda", dtype=torch.int32), 7) == 0)


def test_gradient_behind_32_bits(mrl):
    N, d, V = 525000, 4104, 300                        # dy of 2.15e9 elements
    dy = torch.zeros((N, d), device="cuda", dtype=BF16)
    dy[N - 1] = rand((d,), BF16, 1)
    dy[1] = rand((d,), BF16, 2)
    ids = torch.full((N,), 4, device="cuda", dtype=torch.int32)
    ids[N - 1] = 299
    got = mrl.embedding_backward(dy, ids, V)
    assert torch.equal(got[299], dy[N - 1].float()) and torch.equal(got[4], dy[1].float())
    del dy
    big = torch.empty((530000, d), device="cuda")       # a table of 2.2e9 elements
    rows = rand((2, d), F32, 5)
    mrl.embedding_backward(rows, torch.tensor([529999, 1], device="cuda", dtype=torch.int32), 530000, out=big)
    assert torch.equal(big[529999], rows[0]) and torch.equal(big[1], rows[1]) and torch.all(big[529990:529999] == 0) and torch.all(big[2:9] == 0)


def test_same_bits_again_and_in_a_graph(mrl):
    N, d, V = 9000, 264, 2000
    dy, ids = rand((N, d), BF16, 3), _ids(N, V, 3, 0, 300)
    want = mrl.embedding_backward(dy, ids, V)
    ws = torch.empty(mrl.lib().mrl_embedding_backward_workspace(N, d, V), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(want)
    table = rand((V, d), BF16, 4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            y = mrl.embedding(table, ids)
            mrl.embedding_backward(dy, ids, V, out=out, workspace=ws)
    for k in range(4):
        out.fill_(float("nan"))
        y.zero_()
        ws.random_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(y, table[ids.long()])
        assert torch.equal(mrl.embedding_backward(dy, ids, V), want)
    ids.copy_(_ids(N, V, 9))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, mrl.embedding_backward(dy, ids, V)) and torch.equal(y, table[ids.long()])


def test_gradient_against_differences(mrl):
    """<dy, lookup(table)> is linear in the table: its difference along a direction is the gradient's product with it, to rounding."""
    N, d, V = 200, 24, 30
    t, e, dy, ids = rand((V, d), F32, 1), rand((V, d), F32, 2), rand((N, d), F32, 3), _ids(N, V, 4)
    f = lambda x: float((mrl.embedding(x, ids, 1.5).double() * dy.double()).sum())
    step = 0.5
    diff = (f(t + step * e) - f(t - step * e)) / (2 * step)
    got = float((mrl.embedding_backward(dy, ids, V, 1.5).double() * e.double()).sum())
    # 4800 products with a rounding or two of U of values below 10 each, over the step
    assert abs(diff - got) <= 4800 * 4 * U * 10 / step
