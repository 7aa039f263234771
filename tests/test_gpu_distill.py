"""Distillation loss through the head, forward and backward, against 64 bits, where it can go wrong.

Bounds.  U = 2^-24 is half a step of fp32.  A logit is a sum of d products, at most d roundings of partial sums no larger than A = sum |h w|, so that it is off by
d U A / T at most, and a log-prob by twice that (with the log-sum-exp); exponents in the log2 domain are rounded at the size of |z / T| and the margin of 60: (4 |z| / T + 120) U,
the sums of V exponentials to (V / 128 + 150) U.  The divergence is a sum of those with weights q, and never worse than the 2e-3 that log-probs are held to elsewhere.
Gradients of the bf16 path: operands rounded to 2^-9 of themselves at random; the bounds of the other loss (1e-2 in the whole, per row 2e-2) apply.  Gradients of
the fp32 path: 2e-4 as there."""
import numpy as np
import pytest
import torch

from tests import top_oracle as to
from tests import util
from tests.top_oracle import f64, rand

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def mrl():
    import paper_2605_07244_amd as m
    m.lib()
    return m


def _case(N, d, V, k, dtype, seed, T=1.0, scale=2.0):
    """A student and alternatives of a teacher near it; some ids are none."""
    h, w = rand((N, d), dtype, seed), rand((V, d), dtype, seed + 1, scale / d ** 0.5)
    z = (h.float() + 0.5 * rand((N, d), F32, seed + 2)) @ w.float().t() / T
    if k <= V:
        ids = z.topk(k, dim=1).indices.int()
    else:
        ids = torch.randint(0, V, (N, k), device="cuda", dtype=torch.int32, generator=torch.Generator("cuda").manual_seed(seed))
    logp = (z - z.logsumexp(1, keepdim=True)).gather(1, ids.long()).contiguous()
    g = torch.Generator("cuda").manual_seed(seed + 3)
    ids = torch.where(torch.rand(N, k, device="cuda", generator=g) < 0.1, -1, ids).contiguous()
    if k > 0:
        ids[:, 0] = ids[:, 0].clamp(min=0)
    return h, w, ids, logp


def _kl_bound(h, w, T, V, mass):
    """Per row."""
    h64, w64 = np.abs(f64(h)), np.abs(f64(w))
    A = (h64 @ w64.T).max(1)
    z = np.abs(f64(h) @ f64(w).T).max(1)
    d = h.shape[1]
    return np.minimum(2e-3, 2 * d * U * A / T + (4 * z / T + 120 + V / 128 + 150) * U) * np.maximum(mass, 1e-3) + 2 * U


def _check(mrl, h, w, ids, logp, cfg, mask=None, weight=None, base=None, workspace=None, grads=True, kl_slack=0.0):
    dw = None if base is None else base.clone()
    r = mrl.distill_loss_fwd_bwd(h, w, ids, logp, cfg, token_mask=mask, row_weight=weight, out_dW=dw, workspace=workspace, want_dH=grads, want_dW=grads)
    torch.cuda.synchronize()
    m = None if mask is None else mask.cpu().numpy()
    wt = None if weight is None else f64(weight)
    h64 = f64(h) if m is None else np.where(m[:, None] != 0, f64(h), 0.0)
    lp = f64(logp) if m is None else np.where(m[:, None] != 0, f64(logp), 0.0)
    i = ids.cpu().numpy()
    kl, loss, dH, dW = to.distill(h64, f64(w), i, lp, wt, m, cfg.temperature, cfg.renormalize)
    V = w.shape[0]
    there = (i >= 0) & (i < V)
    with np.errstate(all="ignore"):
        q = np.where(there, np.exp(np.where(there, lp, -np.inf)), 0.0)
        on = (q.sum(1) > 0) if m is None else (q.sum(1) > 0) & (m != 0)
        mass = np.ones(len(kl)) if cfg.renormalize else q.sum(1)
    bound = _kl_bound(torch.from_numpy(h64), w, cfg.temperature, V, mass) + kl_slack
    err = np.abs(f64(r["kl"]) - kl)
    print(f"kl: worst error over its bound {float(np.max(err / bound)):.3f}, {float(err.max()):.2e}")
    assert np.all(err <= bound) and np.all(f64(r["kl"])[~on] == 0)
    st = mrl.read_distill_stats(r["stats"])
    assert st["n_scored_rows"] == on.sum() and st["n_saturated_rows"] == 0
    assert st["n_empty_rows"] == ((m != 0) if m is not None else np.ones(len(on), bool)).sum() - on.sum()
    assert st["n_bad_ids"] == (i[on] >= V).sum()
    c = np.where(on, np.full(len(on), 1 / max(1, on.sum())) if wt is None else wt, 0.0)
    T2 = cfg.temperature ** 2
    assert abs(st["loss_total"] - loss) <= T2 * float(np.sum(np.abs(c) * (bound + 2 * U * np.abs(kl)))) + 1e-12
    if not grads:
        assert r["dH"] is None and r["dW"] is None
        return r, st
    tol = util.F32_REL_TOL if h.dtype == F32 else util.REL_TOL
    util.check_gradient("dH", f64(r["dH"]), dH, tol)
    got = f64(r["dW"]) - (0.0 if base is None else f64(base))
    if base is not None:
        # the sum with what was there is rounded to fp32
        assert np.linalg.norm(got - dW) <= tol * np.linalg.norm(dW) + U * np.linalg.norm(f64(r["dW"]))
    else:
        util.check_gradient("dW", got, dW, tol)
    assert torch.all(r["dH"][torch.from_numpy(~on).cuda()] == 0)
    return r, st


SHAPES = [(1, 64, 2, 1), (1, 128, 300, 256), (3, 136, 700, 7), (40, 256, 1000, 64), (200, 96, 5003, 255), (257, 384, 2500, 20), (700, 712, 1031, 65), (1500, 128, 513, 33),
          (4200, 64, 300, 5), (17, 1536, 50257, 50)]


@pytest.mark.parametrize("N,d,V,k", SHAPES)
def test_sizes(mrl, N, d, V, k):
    h, w, ids, logp = _case(N, d, V, k, BF16, N + d)
    _check(mrl, h, w, ids, logp, mrl.DistillConfig())


@pytest.mark.parametrize("T", [0.5, 2.0, 7.0])
@pytest.mark.parametrize("renormalize", [0, 1])
@pytest.mark.parametrize("dh,dw", [(0, 0), (1, 1), (1, 0)])
def test_options(mrl, T, renormalize, dh, dw):
    N, d, V, k = 300, 200, 1500, 40
    h, w, ids, logp = _case(N, d, V, k, BF16, 5, T)
    weight = torch.rand(N, device="cuda", generator=torch.Generator("cuda").manual_seed(1)) / N
    weight[3] = 0.0
    weight[4] = -weight[4]
    mask = (torch.arange(N, device="cuda") % 3 != 0).to(torch.uint8)
    _check(mrl, h, w, ids, logp, mrl.DistillConfig(temperature=T, renormalize=renormalize, dh_dtype=dh, dw_dtype=dw), mask, weight)
    _check(mrl, h, w, ids, logp, mrl.DistillConfig(temperature=T, renormalize=renormalize, dh_dtype=dh, dw_dtype=dw), grads=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,scale", [(0.01, 0.02), (0.1, 0.2), (100.0, 100.0), (100.0, 2.0)])
@pytest.mark.parametrize("renormalize", [0, 1])
def test_temperatures_at_the_ends_of_the_range(mrl, dtype, T, scale, renormalize):
    h, w, ids, logp = _case(300, 136, 900, 12, dtype, 5, T, scale)
    _check(mrl, h, w, ids, logp, mrl.DistillConfig(temperature=T, renormalize=renormalize, dh_dtype=mrl.F32))


@pytest.mark.parametrize("N,d,V,k", [(1, 1, 1, 1), (5, 3, 7, 3), (64, 64, 512, 16), (300, 50, 2100, 100), (4100, 8, 33, 5), (9, 100, 5000, 256)])
@pytest.mark.parametrize("T,renormalize", [(1.0, 1), (3.0, 0)])
def test_fp32(mrl, N, d, V, k, T, renormalize):
    h, w, ids, logp = _case(N, d, V, k, F32, N + d, T)
    mask = (torch.arange(N, device="cuda") % 4 != 3).to(torch.uint8)
    cfg = mrl.DistillConfig(temperature=T, renormalize=renormalize, dh_dtype=mrl.F32)
    _check(mrl, h, w, ids, logp, cfg, mask)
    _check(mrl, h, w, ids, logp, cfg, mask, grads=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dw", [0, 1])
def test_passes(mrl, dtype, dw):
    """Several passes, some without rows; gradients are added over them, and into what was there."""
    N, d, V, k = 2000, 136, 900, 30
    h, w, ids, logp = _case(N, d, V, k, dtype, 9)
    mask = (torch.arange(N, device="cuda") < 900).to(torch.uint8)
    if dtype == F32 and dw:
        return
    dh = mrl.F32 if dtype == F32 else mrl.BF16
    for m in (None, mask):
        a, _ = _check(mrl, h, w, ids, logp, mrl.DistillConfig(dh_dtype=dh, dw_dtype=dw, chunk_rows=256), m)
        b, _ = _check(mrl, h, w, ids, logp, mrl.DistillConfig(dh_dtype=dh, dw_dtype=dw), m)
        assert torch.equal(a["kl"], b["kl"])
    if not dw:
        base = rand((V, d), F32, 77, 1e-4)
        _check(mrl, h, w, ids, logp, mrl.DistillConfig(dh_dtype=dh, accumulate_dw=1, chunk_rows=512), mask, base=base)
        _check(mrl, h, w, ids, logp, mrl.DistillConfig(dh_dtype=dh, accumulate_dw=1), base=base)


@pytest.mark.parametrize("N,scored,d,V,chunk_rows,cut", [
    (200, 200, 1536, 5000, 0, None),                    # a launch for few rows, whole lines of dW
    (900, 577, 712, 1031, 0, None),                     # ... lines that straddle, ragged tiles
    (300, 0, 136, 700, 0, None),                        # ... without a row
    (1280, 1, 1024, 16405, 1280, (0, 65, 0, 4, 8)),     # tiles of 256 with a tail of slices, most of them empty
    (1280, 327, 1024, 16405, 1280, (0, 65, 0, 4, 8)),
    (1280, 0, 1024, 16405, 1280, (0, 65, 0, 4, 8)),
    (1536, 1400, 1536, 11000, 0, (0, 43, 0, 18, 8)),
    (4200, 4200, 1032, 24000, 0, (0, 94, 0, 30, 2)),
    (2000, 2000, 136, 1000, 0, (3, 0, 0, 3, 4)),        # tiles of 384, all of them in slices
    (2000, 0, 136, 1000, 0, (3, 0, 0, 3, 1)),
    (2000, 2000, 3080, 9999, 0, (27, 0, 0, 95, 2)),     # a whole round and slices
    (3500, 3400, 2056, 21000, 0, (55, 0, 0, 239, 1)),
])
def test_bf16_gradient_of_the_head_is_the_float_one_rounded(mrl, N, scored, d, V, chunk_rows, cut):
    """Each of the launches of dW with a bf16 output: the bits of the float output, rounded once; scratch that holds NaN before."""
    h, w = rand((N, d), BF16, N), rand((V, d), BF16, N + 1, 2.0 / d ** 0.5)
    g = torch.Generator("cuda").manual_seed(N)
    ids = torch.randint(0, V, (N, 9), device="cuda", generator=g, dtype=torch.int32)
    logp = -3 * torch.rand(N, 9, device="cuda", generator=g)
    mask = (torch.randperm(N, device="cuda", generator=g) < scored).to(torch.uint8)
    chunk = chunk_rows or -(-N // 256) * 256
    if cut is None:
        assert N <= mrl.dw_few_rows()
    else:
        c = mrl.gemm_cut(mrl.GEMM_DW, max(scored, 1), V, d, chunk, min(N, chunk))
        assert (c["wide"], c["narrow"], c["half"], c["rest"]) == cut[:4] and (scored == 0 or c["split"] == cut[4])
    out = []
    for dw in (mrl.F32, mrl.BF16):
        cfg = mrl.DistillConfig(dw_dtype=dw, chunk_rows=chunk_rows)
        ws = torch.full((mrl.distill_loss_workspace(N, d, V, 9, mrl.BF16, cfg),), 255, dtype=torch.uint8, device="cuda")
        dW = torch.full((V + 1, d), float("nan"), device="cuda", dtype=F32 if dw == mrl.F32 else BF16)
        out.append(mrl.distill_loss_fwd_bwd(h, w, ids, logp, cfg, token_mask=mask, out_dW=dW[:V], workspace=ws))
        assert torch.all(torch.isnan(dW[V].float()))    # (nothing behind the last row)
    a, b = out
    assert torch.equal(a["dW"].bfloat16(), b["dW"]) and torch.equal(a["dH"], b["dH"]) and torch.equal(a["kl"], b["kl"])
    if scored == 0:
        assert torch.all(a["dW"] == 0) and torch.all(b["dW"] == 0)
    else:
        # column sums of dz are zero: so are those of dW's rows, to its operands' rounding
        assert float(a["dW"].double().sum(0).abs().max()) <= 2.0 ** -7 * float(a["dW"].double().abs().sum(0).max())


@pytest.mark.parametrize("N,d,V", [(100, 2048, 66001), (700, 1032, 110000)])
def test_bf16_gradient_of_a_large_head_and_few_rows(mrl, N, d, V):
    """Heads of 2048 tiles and more take the large tiles for few rows too, with a bf16 gradient: another order of the same products than the float one's launch."""
    h, w = rand((N, d), BF16, N), rand((V, d), BF16, N + 1, 2.0 / d ** 0.5)
    ids = torch.randint(0, V, (N, 5), device="cuda", generator=torch.Generator("cuda").manual_seed(N), dtype=torch.int32)
    logp = torch.full((N, 5), -1.0, device="cuda")
    a = mrl.distill_loss_fwd_bwd(h, w, ids, logp, mrl.DistillConfig())
    ws = torch.full((mrl.distill_loss_workspace(N, d, V, 5, mrl.BF16, mrl.DistillConfig(dw_dtype=mrl.BF16)),), 255, dtype=torch.uint8, device="cuda")
    b = mrl.distill_loss_fwd_bwd(h, w, ids, logp, mrl.DistillConfig(dw_dtype=mrl.BF16), workspace=ws)
    assert torch.equal(a["dH"], b["dH"]) and torch.equal(a["kl"], b["kl"])
    # N products, each partial sum rounded, of at most the sum of their magnitudes: that of column k is below the sum of |h| times the largest scaled exponential's share
    mag = 2.0 / N * h.float().abs().sum(0)
    assert torch.all((a["dW"] - b["dW"].float()).abs() <= 2.0 ** -8 * a["dW"].abs() + 2 * N * U * mag)


@pytest.mark.parametrize("N,scored,d,V", [
    (1, 1, 8, 1), (32, 32, 264, 63), (33, 33, 712, 64), (70, 64, 1536, 1000), (100, 100, 256, 20011), (130, 128, 136, 70001), (140, 129, 1032, 4097),
    (192, 161, 4096, 3001), (200, 200, 1536, 9999), (225, 225, 2056, 5003), (256, 256, 3080, 12345), (256, 0, 520, 777), (200, 0, 2048, 30000),
    (256, 250, 16384, 500), (256, 250, 16392, 300), (20, 20, 64, 151936),
    (60, 50, 72, 400003), (256, 240, 328, 151936), (30, 30, 712, 60000),   # widths whose last wave has half its columns, and skips half the stores of floats
    (200, 190, 8, 3000001)])                            # (blocks that read the stash take several pieces of a row)
def test_gradient_of_the_head_of_up_to_256_rows(mrl, N, scored, d, V):
    """Hidden rows in registers: every number of steps, one stage and many of them, ranges of the vocabulary that end beside it, widths beside the waves'."""
    h, w = rand((N, d), BF16, N), rand((V, d), BF16, N + 1, 2.0 / d ** 0.5)
    g = torch.Generator("cuda").manual_seed(N)
    ids = torch.randint(0, V, (N, 7), device="cuda", generator=g, dtype=torch.int32)
    logp = -3 * torch.rand(N, 7, device="cuda", generator=g)
    mask = (torch.randperm(N, device="cuda", generator=g) < scored).to(torch.uint8)
    out = []
    for dw in (mrl.F32, mrl.BF16, mrl.BF16):
        cfg = mrl.DistillConfig(dw_dtype=dw)
        ws = torch.full((mrl.distill_loss_workspace(N, d, V, 7, mrl.BF16, cfg),), 255, dtype=torch.uint8, device="cuda")
        dW = torch.full((V + 2, d), float("nan"), device="cuda", dtype=F32 if dw == mrl.F32 else BF16)
        r = mrl.distill_loss_fwd_bwd(h, w, ids, logp, cfg, token_mask=mask, out_dW=dW[1:V + 1], want_dH=len(out) < 2, workspace=ws)
        assert torch.all(torch.isnan(dW[0].float())) and torch.all(torch.isnan(dW[V + 1].float()))
        out.append(r)
    a, b, c = out
    assert torch.equal(a["dW"].bfloat16(), b["dW"]) and torch.equal(b["dW"], c["dW"]) and torch.equal(a["dH"], b["dH"]) and torch.equal(a["kl"], c["kl"])
    assert scored > 0 or torch.all(b["dW"] == 0)
    # the launch that adds into a float dW, of nothing: the same products in the same order
    r = mrl.distill_loss_fwd_bwd(h, w, ids, logp, mrl.DistillConfig(accumulate_dw=1), token_mask=mask, out_dW=torch.zeros(V, d, device="cuda"), want_dH=False)
    assert torch.equal(r["dW"], a["dW"])


def test_bf16_gradient_at_any_address(mrl):
    N, d, V = 1500, 136, 900
    h, w, ids, logp = _case(N, d, V, 7, BF16, 3)
    for n in (N, 200):
        args = (h[:n].contiguous(), w, ids[:n].contiguous(), logp[:n].contiguous())
        want = mrl.distill_loss_fwd_bwd(*args, mrl.DistillConfig(dw_dtype=mrl.BF16))
        buf = torch.zeros(V * d + 3, device="cuda", dtype=BF16)
        got = mrl.distill_loss_fwd_bwd(*args, mrl.DistillConfig(dw_dtype=mrl.BF16), out_dW=buf[1:1 + V * d].view(V, d))
        assert torch.equal(got["dW"], want["dW"]) and buf[0] == 0 and torch.all(buf[1 + V * d:] == 0)


def test_smaller_workspace(mrl):
    N, d, V, k = 3000, 128, 1000, 20
    h, w, ids, logp = _case(N, d, V, k, BF16, 4)
    cfg = mrl.DistillConfig()
    need = mrl.distill_loss_workspace(N, d, V, k, mrl.BF16, mrl.DistillConfig(chunk_rows=512))
    assert need < mrl.distill_loss_workspace(N, d, V, k, mrl.BF16, cfg)
    _check(mrl, h, w, ids, logp, cfg, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"))
    with pytest.raises(mrl.MrlError):
        mrl.distill_loss_fwd_bwd(h, w, ids, logp, cfg, workspace=torch.empty(100000, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k", [9, 130])
def test_ids_listed_twice_and_no_ids(mrl, dtype, k):
    N, d, V = 80, 64, 150
    h, w, ids, logp = _case(N, d, V, k, dtype, 3)
    ids[0] = 7                                          # one id, k times
    ids[1, 1::2] = ids[1, 0]
    ids[2, k - 1] = ids[2, 0]
    ids[3] = -1                                         # none
    ids[4] = V
    ids[5, 1:] = 2 ** 31 - 1
    ids[6, ::2] = -2 ** 31
    logp[7] = -float("inf")
    logp[8, 1:] = -float("inf")
    logp[9, 0] = -float("inf")
    logp[10, 1:] = -700.0
    cfg = dict(dh_dtype=mrl.F32)
    for renormalize in (0, 1):
        r, st = _check(mrl, h, w, ids, logp, mrl.DistillConfig(renormalize=renormalize, **cfg))
        assert st["n_empty_rows"] == 3 and st["n_bad_ids"] == k - 1
    # rows without alternatives only
    r = mrl.distill_loss_fwd_bwd(h, w, torch.full_like(ids, -1), logp, mrl.DistillConfig(**cfg))
    st = mrl.read_distill_stats(r["stats"])
    assert st["n_scored_rows"] == 0 and st["loss_total"] == 0 and torch.all(r["dH"] == 0) and torch.all(r["dW"] == 0) and torch.all(r["kl"] == 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masked_rows_are_not_read(mrl, dtype):
    N, d, V, k = 300, 72, 400, 12
    h, w, ids, logp = _case(N, d, V, k, dtype, 8)
    mask = (torch.arange(N, device="cuda") % 2).to(torch.uint8)
    h[::2] = float("nan")
    logp[::2] = float("nan")
    ids[::2] = 2 ** 30
    r, _ = _check(mrl, h, w, ids, logp, mrl.DistillConfig(dh_dtype=mrl.F32), mask)
    assert torch.all(torch.isfinite(r["dW"]))
    r = mrl.distill_loss_fwd_bwd(h, w, ids, logp, mrl.DistillConfig(dh_dtype=mrl.F32), token_mask=torch.zeros_like(mask))
    assert torch.all(r["dW"] == 0) and torch.all(r["dH"] == 0) and mrl.read_distill_stats(r["stats"])["n_empty_rows"] == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_nan_stays_in_its_row_of_dH(mrl, dtype):
    N, d, V, k = 40, 64, 300, 6
    h, w, ids, logp = _case(N, d, V, k, dtype, 8)
    want = mrl.distill_loss_fwd_bwd(h, w, ids, logp, mrl.DistillConfig(dh_dtype=mrl.F32))
    logp[5, 0] = float("nan")
    logp[6] = float("nan")
    h[7, 3] = float("nan")
    r = mrl.distill_loss_fwd_bwd(h, w, ids, logp, mrl.DistillConfig(dh_dtype=mrl.F32))
    bad = torch.zeros(N, dtype=torch.bool, device="cuda")
    bad[5:8] = True
    assert torch.equal(torch.isnan(r["kl"]), bad) and torch.equal(r["kl"][~bad], want["kl"][~bad])
    assert torch.equal(torch.isnan(r["dH"]).any(1), bad)
    assert torch.isnan(r["dW"]).any() and np.isnan(mrl.read_distill_stats(r["stats"])["loss_total"])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k", [1, 63, 64, 128, 256])
@pytest.mark.parametrize("renormalize", [0, 1])
def test_log_probs_that_are_all_nan_count(mrl, dtype, k, renormalize):
    """Every lane of the wave that looks at them holds NaN, at 64 alternatives and multiples; a NaN is no empty row."""
    N, d, V = 12, 64, 300
    h, w, ids, logp = _case(N, d, V, k, dtype, 8)
    ids.clamp_(min=0)
    logp[5] = float("nan")
    r = mrl.distill_loss_fwd_bwd(h, w, ids, logp, mrl.DistillConfig(renormalize=renormalize, dh_dtype=mrl.F32))
    st = mrl.read_distill_stats(r["stats"])
    bad = torch.arange(N, device="cuda") == 5
    assert torch.equal(torch.isnan(r["kl"]), bad) and torch.equal(torch.isnan(r["dH"]).any(1), bad)
    assert torch.isnan(r["dW"]).any() and np.isnan(st["loss_total"]) and st["n_scored_rows"] == N and st["n_empty_rows"] == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("renormalize", [0, 1])
def test_infinite_log_probs_are_nan(mrl, dtype, renormalize):
    N, d, V, k = 12, 64, 300, 6
    h, w, ids, logp = _case(N, d, V, k, dtype, 8)
    logp[5, 0] = float("inf")
    ids[6], logp[6] = 7, float("inf")
    r = mrl.distill_loss_fwd_bwd(h, w, ids, logp, mrl.DistillConfig(renormalize=renormalize, dh_dtype=mrl.F32))
    bad = (torch.arange(N, device="cuda") - 5).div(2, rounding_mode="floor") == 0
    assert torch.equal(torch.isnan(r["kl"]), bad) and torch.equal(torch.isnan(r["dH"]).any(1), bad) and torch.all(torch.isfinite(r["kl"][~bad]))
    assert torch.isnan(r["dW"]).any() and np.isnan(mrl.read_distill_stats(r["stats"])["loss_total"])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("given", [-20.0, -45.0, -65.0])
@pytest.mark.parametrize("seen", [60.0, 75.0, 95.0])
def test_small_masses_of_ids_that_the_student_rules_out(mrl, dtype, given, seen):
    """Masses down to e^-65 beside sums of exponentials e^seen times the id's own: their quotient and the row's scale are beyond fp32, the gradient is not."""
    N, d, V = 20, 64, 300
    h, w = rand((N, d), dtype, 1, 0.3), rand((V, d), dtype, 2, 0.1)
    h[:, 0], w[:, 0] = seen, 0.0
    w[5, 0] = 1.0                                       # the student's token, with a logit of `seen` more than the others
    ids = torch.full((N, 1), 9, device="cuda", dtype=torch.int32)
    logp = torch.full((N, 1), given, device="cuda")
    for dh in (mrl.F32, mrl.BF16) if dtype == BF16 else (mrl.F32,):
        r = mrl.distill_loss_fwd_bwd(h, w, ids, logp, mrl.DistillConfig(renormalize=0, dh_dtype=dh))
        kl, loss, dH, dW = to.distill(f64(h), f64(w), ids.cpu().numpy(), f64(logp), renormalize=False)
        # a log-prob is off by twice what a logit is, d roundings at the sum of its products' magnitudes, and by the exponents' and sums' roundings
        A = (np.abs(f64(h)) @ np.abs(f64(w)).T).max()
        off = 2 * d * U * A + (4 * A + 120 + V / 128 + 150) * U
        assert np.all(np.abs(f64(r["kl"]) - kl) <= np.exp(given) * off + 2 * U * np.abs(kl))
        st = mrl.read_distill_stats(r["stats"])
        assert st["n_saturated_rows"] == 0 and st["n_scored_rows"] == N and abs(st["loss_total"] - loss) <= np.exp(given) * off + 2 * U * abs(loss)
        tol = util.F32_REL_TOL if dtype == F32 else util.REL_TOL
        for name, got, want in (("dH", r["dH"], dH), ("dW", r["dW"], dW)):
            util.check_gradient(name, f64(got), want, tol)


@pytest.mark.parametrize("N", [40, 300])
def test_a_row_of_small_mass_among_others(mrl, N):
    d, V, k = 64, 300, 7
    h, w, ids, logp = _case(N, d, V, k, BF16, 4, scale=1.0)
    h[7] = (70.0 * w[5].float() / w[5].float().square().sum()).bfloat16()      # the student's token is 5, by 70 more than what it sees none of
    z = (h[7].float() @ w.float().t()).cpu()
    ids[7] = -1
    ids[7, 0] = int(z.abs().argmin())
    logp[7, 0] = -65.0
    r = mrl.distill_loss_fwd_bwd(h, w, ids, logp, mrl.DistillConfig(renormalize=0, dh_dtype=mrl.F32))
    _, _, dH, dW = to.distill(f64(h), f64(w), ids.cpu().numpy(), f64(logp), renormalize=False)
    assert mrl.read_distill_stats(r["stats"])["n_saturated_rows"] == 0
    util.check_gradient("dW", f64(r["dW"]), dW)
    util.check_gradient("dH", f64(r["dH"]), dH)
    util.check_gradient("dH of the row", f64(r["dH"])[7:8], dH[7:8])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,V", [(40, 300), (300, 700), (600, 5003)])
@pytest.mark.parametrize("grads", [True, False])
def test_nan_and_infinities_in_the_head(mrl, dtype, N, V, grads):
    """... in a row that no alternative names: the softmax of every row that it makes NaN or +infinite is NaN, and of no other."""
    d, k, v = 64, 6, V - 7
    h, w, ids, logp = _case(N, d, V, k, dtype, 8)
    ids[ids == v] = -1
    ids[:, 0] = torch.where(ids[:, 0] < 0, 3, ids[:, 0])
    h[:, 3] = torch.where(torch.arange(N, device="cuda") % 3 == 0, 1.0, -0.5)
    cfg = mrl.DistillConfig(dh_dtype=mrl.F32)
    for value in (float("nan"), float("inf"), -float("inf")):
        w[v, 3] = value
        r = mrl.distill_loss_fwd_bwd(h, w, ids, logp, cfg, want_dH=grads, want_dW=grads)
        st = mrl.read_distill_stats(r["stats"])
        bad = torch.isnan(h[:, 3] * value) | (h[:, 3] * value > 0)
        assert torch.equal(torch.isnan(r["kl"]), bad), value
        assert np.isnan(st["loss_total"]) and st["n_scored_rows"] == N and st["n_saturated_rows"] == 0
        # the others: the token's probability is 0
        rest = torch.cat([w[:v], w[v + 1:]])
        i = torch.where(ids > v, ids - 1, ids)
        want, _, _, _ = to.distill(f64(h), f64(rest), i.cpu().numpy(), f64(logp))
        ok = (~bad).cpu().numpy()
        bound = _kl_bound(h, rest, 1.0, V, np.ones(N))
        assert np.all(np.abs(f64(r["kl"]) - want)[ok] <= bound[ok])
        if grads:
            assert torch.isnan(r["dW"]).any() and torch.all(torch.isnan(r["dH"][bad]).any(1))


def test_saturated_rows_are_counted_and_left_out(mrl):
    N, d, V = 20, 64, 200
    h = torch.zeros(N, d, device="cuda", dtype=BF16)
    w = torch.zeros(V, d, device="cuda", dtype=BF16)
    h[:, 0] = 16.0
    w[5, 0] = 10.0                                      # a logit of 160 against zeros
    ids = torch.full((N, 2), 5, device="cuda", dtype=torch.int32)
    ids[:, 1] = 6
    ids[3:6, 0] = 9                                     # alternatives that the student rules out
    logp = torch.full((N, 2), -0.7, device="cuda")
    r = mrl.distill_loss_fwd_bwd(h, w, ids, logp, mrl.DistillConfig())
    st = mrl.read_distill_stats(r["stats"])
    assert st["n_saturated_rows"] == 3 and st["n_scored_rows"] == N
    assert torch.all(r["dH"][3:6] == 0) and torch.all(torch.isfinite(r["kl"])) and torch.all(r["kl"][3:6] > 80)
    kl, _, dH, _ = to.distill(f64(h), f64(w), ids.cpu().numpy(), f64(logp))
    ok = np.r_[0:3, 6:N]
    assert np.allclose(f64(r["kl"])[ok], kl[ok], rtol=1e-5)
    assert abs(st["loss_total"] - kl[ok].sum() / N) <= 1e-4 * kl.sum()
    util.check_gradient("dH", f64(r["dH"])[ok], dH[ok])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_alternative_is_the_likelihood(mrl, dtype):
    """k = 1: the negative log-prob of the id, as the scoring pass has it."""
    N, d, V = 300, 128, 2000
    h, w, ids, logp = _case(N, d, V, 1, dtype, 6)
    r = mrl.distill_loss_fwd_bwd(h, w, ids, logp, mrl.DistillConfig(dh_dtype=mrl.F32), want_dW=False)
    lp, _ = mrl.token_logprobs(h, w, ids[:, 0].contiguous())
    assert r["dW"] is None and torch.allclose(r["kl"], -lp, rtol=0, atol=2e-5)


def test_logits_of_any_size(mrl):
    """Offsets and scales of the logits that a softmax does not see."""
    N, d, V, k = 60, 64, 800, 10
    h, w, ids, logp = _case(N, d, V, k, BF16, 2, scale=1.0)
    h[:, 0], w[:, 0] = 64.0, 50.0                       # 3200 added to every logit: exact in bf16
    r = mrl.distill_loss_fwd_bwd(h, w, ids, logp, mrl.DistillConfig())
    kl, _, dH, dW = to.distill(f64(h), f64(w), ids.cpu().numpy(), f64(logp))
    # partial sums of 3200 are rounded to 2^-12 of one at most 64 times over
    assert np.max(np.abs(f64(r["kl"]) - kl)) <= 2 * 64 * 3300 * U
    # dz's entries are rounded to bf16, by half a step of 2^-8 of themselves at most, and their p is off by twice what a logit is; each goes into dH times its
    # entry of w, 50 in the column whose exact gradient is 0 (sum_v dz_v = 0), where no relative bound can hold
    z64 = f64(h) @ f64(w).T
    p64 = np.exp(z64 - z64.max(1, keepdims=True))
    p64 /= p64.sum(1, keepdims=True)
    i, lp = ids.cpu().numpy(), f64(logp)
    q64 = np.where(i >= 0, np.exp(lp), 0.0)
    q64 /= q64.sum(1, keepdims=True)
    dz = p64.copy()
    for n in range(N):
        np.subtract.at(dz[n], i[n][i[n] >= 0], q64[n][i[n] >= 0])
    off = (2.0 ** -8 * np.abs(dz) + 2 * 64 * 3300 * U * p64) / N @ np.abs(f64(w))
    assert np.all(np.abs(f64(r["dH"]) - dH) <= off + 2.0 ** -8 * np.abs(dH))


def test_gradient_against_differences(mrl):
    N, d, V, k, T = 24, 16, 40, 6, 1.5
    h, w, ids, logp = _case(N, d, V, k, F32, 12, T)
    cfg = mrl.DistillConfig(temperature=T, renormalize=0, dh_dtype=mrl.F32)
    r = mrl.distill_loss_fwd_bwd(h, w, ids, logp, cfg)
    eh, ew = rand((N, d), F32, 1), rand((V, d), F32, 2, 0.3)
    args = (ids.cpu().numpy(), f64(logp), None, None, T, False)
    f = lambda s: to.distill(f64(h) + s * f64(eh), f64(w) + s * f64(ew), *args)[1]
    step = 1e-5
    diff = (f(step) - f(-step)) / (2 * step)
    got = float(np.sum(f64(r["dH"]) * f64(eh)) + np.sum(f64(r["dW"]) * f64(ew)))
    assert abs(diff - got) <= 2e-4 * (np.sum(np.abs(f64(r["dH"]) * f64(eh))) + np.sum(np.abs(f64(r["dW"]) * f64(ew))))
    # and the kernel's own loss
    loss = lambda s: mrl.read_distill_stats(mrl.distill_loss_fwd_bwd((h + s * eh), (w + s * ew), ids, logp, cfg, want_dH=False, want_dW=False)["stats"])["loss_total"]
    step = 2.0 ** -6
    own = (loss(step) - loss(-step)) / (2 * step)
    # the third derivative's share, from the exact function, and kl's rounding over the step
    exact = (f(step) - f(-step)) / (2 * step)
    assert abs(own - exact) <= T * T * 2e-5 / step


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N", [700, 200])
def test_same_bits_again_and_in_a_graph(mrl, N, dtype):
    d, V, k = 136, 1100, 20
    h, w, ids, logp = _case(N, d, V, k, dtype, 3)
    mask = (torch.arange(N, device="cuda") % 3 != 0).to(torch.uint8)
    cfg = mrl.DistillConfig(dh_dtype=mrl.F32 if dtype == F32 else mrl.BF16, dw_dtype=mrl.BF16 if dtype == BF16 and N == 200 else mrl.F32)
    want = mrl.distill_loss_fwd_bwd(h, w, ids, logp, cfg, token_mask=mask)
    dt = mrl.F32 if dtype == F32 else mrl.BF16
    ws = torch.empty(mrl.distill_loss_workspace(N, d, V, k, dt, cfg), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            got = mrl.distill_loss_fwd_bwd(h, w, ids, logp, cfg, token_mask=mask, workspace=ws)
    for _ in range(4):
        for name in ("kl", "dH", "dW"):
            got[name].fill_(float("nan"))
        ws.random_()
        graph.replay()
        torch.cuda.synchronize()
        eager = mrl.distill_loss_fwd_bwd(h, w, ids, logp, cfg, token_mask=mask)
        for name in ("kl", "dH", "dW", "stats"):
            assert torch.equal(got[name], want[name]) and torch.equal(eager[name], want[name]), name


@pytest.mark.parametrize("N", [600, 100])
def test_two_streams(mrl, N):
    cases = [_case(N, 256, 3000, 16, BF16, s) for s in (1, 2)]
    want = [mrl.distill_loss_fwd_bwd(*c, mrl.DistillConfig()) for c in cases]
    torch.cuda.synchronize()
    got = []
    for c in cases:
        with torch.cuda.stream(torch.cuda.Stream()):
            got.append([mrl.distill_loss_fwd_bwd(*c, mrl.DistillConfig()) for _ in range(3)])
    torch.cuda.synchronize()
    for g, x in zip(got, want):
        for r in g:
            assert all(torch.equal(r[n], x[n]) for n in ("kl", "dH", "dW", "stats"))


def test_a_training_step_from_ids_to_the_tied_weight(mrl):
    """Embedding, norm, a teacher's alternatives, distillation, and back, all gradients of the table in one buffer, then its update."""
    N, d, V, k, T, eps = 200, 128, 900, 24, 2.0, 1e-6
    g = torch.Generator("cuda").manual_seed(0)
    table = rand((V, d), F32, 1, 0.3)
    copy = table.bfloat16()
    gain = torch.rand(d, device="cuda", generator=g) + 0.5
    ids = torch.randint(0, 60, (N,), device="cuda", generator=g, dtype=torch.int32)
    mask = (torch.arange(N, device="cuda") % 5 != 4).to(torch.uint8)
    teacher = rand((N, V), BF16, 5, 2.0)

    top = mrl.top_logprobs(teacher, k, token_mask=mask, temperature=T)
    x = mrl.embedding(copy, ids, d ** 0.5, mask)
    h, _, _ = mrl.rms_norm(x, gain, eps, token_mask=mask)
    cfg = mrl.DistillConfig(temperature=T, dh_dtype=mrl.F32)
    out = mrl.distill_loss_fwd_bwd(h, copy, top["ids"], top["top_logp"], cfg, token_mask=mask)
    dx, dgain = mrl.rms_norm_backward(out["dH"], x, gain, eps, token_mask=mask, dx_dtype=F32)
    total = mrl.embedding_backward(dx, ids, V, d ** 0.5, mask, out=out["dW"], accumulate=True)
    assert total is out["dW"]
    torch.cuda.synchronize()

    # the same in float64 by autograd, the rounded activations' own gradients passed straight through
    t64 = copy.double().cpu().requires_grad_()
    gain64 = gain.double().cpu().requires_grad_()
    on = mask.cpu().bool()
    xs = t64[ids.cpu().long()] * d ** 0.5
    hs = xs * torch.rsqrt(xs.square().mean(1, keepdim=True) + eps) * gain64
    hs = hs + (h.double().cpu() - hs).detach()
    z = hs @ t64.t() / T
    tl = torch.log_softmax(teacher.double().cpu() / T, 1)
    best = torch.from_numpy(to.top(f64(teacher), k)[0])
    q = torch.softmax(tl.gather(1, best), 1)
    kl = (q * (q.log() - torch.log_softmax(z, 1).gather(1, best))).sum(1)
    loss = T * T * kl[on].mean()
    loss.backward()
    assert abs(mrl.read_distill_stats(out["stats"])["loss_total"] - float(loss)) <= 1e-4 * float(loss)
    util.check_gradient("table", f64(total), t64.grad.numpy())
    assert util.rel_fro(f64(dgain), gain64.grad.numpy()) <= util.REL_TOL

    plan = mrl.adamw_plan([table, gain], [total, dgain], [copy, None])
    before = table.clone()
    mrl.adamw_step(plan, 1e-3, 1, norm_coef=mrl.grad_norm(plan, 1.0))
    torch.cuda.synchronize()
    moved = (table - before).abs()
    assert float(moved.max()) <= 1.1e-3 and torch.equal(copy, table.bfloat16()) and float(moved.mean()) > 1e-4
