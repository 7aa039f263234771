"""Root-mean-square norm and its backward pass against 64 bits, where they can go wrong.

Bounds, from the kernels' sums.  U = 2^-24 is half a step of fp32.  A thread adds at most 64 squares one after the other, the lanes and waves
then at most 10 + 16 sums: the mean is off by at most 90 U of itself, its root and inverse by half of that and two roundings, so
that y's two products leave 50 U.  Outputs of fewer bits add half a step of theirs: 2^-8 of bf16, 2^-4 of e4m3 (2^-10 of a scale below its
smallest normal value)."""
import numpy as np
import pytest
import torch

from tests import update_oracle as uo
from tests.update_oracle import f64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
HALF = {F32: U, BF16: 2.0 ** -8}
EPS = 1e-5
WIDTHS = [1, 2, 7, 8, 9, 15, 16, 63, 64, 65, 71, 100, 128, 129, 136, 255, 256, 257, 512, 513, 712, 1024, 1025, 1536, 2048, 2049, 3584, 4096, 4100, 8191, 8192, 8200, 16384]


@pytest.fixture(scope="module")
def mrl():
    import paper_2605_07244_amd as m
    m.lib()
    return m


def _rand(shape, dtype, seed, scale=1.0):
    g = torch.Generator("cuda").manual_seed(seed)
    return (scale * torch.randn(shape, device="cuda", generator=g)).to(dtype)


def _within(name, got, want, bound):
    err = np.abs(f64(got) - want)
    assert np.all(np.isfinite(err)), name
    worst = float(np.max(err / np.maximum(bound, 1e-300))) if err.size else 0.0
    print(f"{name}: worst error over its bound {worst:.3f}")
    assert np.all(err <= bound), (name, worst)


def _check_forward(mrl, x, w, residual=None, mask=None, out=None, block=0):
    y, h, scale = mrl.rms_norm(x, w, EPS, residual, mask, out, block)
    torch.cuda.synchronize()
    m = None if mask is None else mask.cpu().numpy()
    want_y, want_h = uo.rms_norm(f64(x), f64(w), EPS, None if residual is None else f64(residual), m)
    assert (h is None) == (residual is None) and y.dtype == (out or x.dtype)
    if h is not None:
        # the sum of two fp32 numbers is rounded once, and once more to h's type
        _within("h", h, want_h, (HALF[h.dtype] + U) * np.abs(want_h))
    # h enters y with the rounding of the sum, relative to the sum itself
    if y.dtype != E4M3:
        assert scale is None
        _within("y", y, want_y, (HALF[y.dtype] + 52 * U) * np.abs(want_y))
        return y, h, scale
    want_s = uo.scales_of(want_y, block)
    got_s = f64(scale).reshape(want_s.shape)
    assert scale.shape == ((x.shape[0], -(-x.shape[1] // block)) if block else (x.shape[0],))
    assert np.all(np.abs(got_s - want_s) <= 54 * U * want_s)
    per = np.repeat(got_s, block or x.shape[1], axis=1)[:, :x.shape[1]]
    # a code stands for y to half a step of e4m3
    err = np.abs(f64(y) * per - want_y)
    assert np.all(err <= (2.0 ** -4 + 60 * U) * np.abs(want_y) + 2.0 ** -10 * per), float(np.max(err))
    top = np.max(np.abs(f64(y)), axis=1)
    live = np.max(np.abs(want_y), axis=1) > 1e-20
    assert np.all(top[live] == 448.0)                              # the largest of a scale takes the largest code
    return y, h, scale


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("N", [1, 5])
def test_forward_widths(mrl, N, d):
    x, w, r = _rand((N, d), BF16, d), 1 + _rand((d,), BF16, d + 1, 0.2), _rand((N, d), BF16, d + 2, 3.0)
    _check_forward(mrl, x, w, r)
    _check_forward(mrl, x, w, r, out=E4M3)
    _check_forward(mrl, x, w, out=E4M3, block=128)
    _check_forward(mrl, x.float(), w.float(), r.float(), out=F32)


@pytest.mark.parametrize("x_type,res_type", [(BF16, None), (BF16, BF16), (BF16, F32), (F32, None), (F32, F32)])
@pytest.mark.parametrize("out,block", [(F32, 0), (BF16, 0), (E4M3, 0), (E4M3, 128)])
@pytest.mark.parametrize("w_type", [BF16, F32])
def test_forward_types(mrl, x_type, res_type, out, block, w_type):
    for N, d in ((1500, 333), (3, 1000), (1030, 1800), (2, 5000)):
        x, w = _rand((N, d), x_type, 1), 1 + _rand((d,), w_type, 2, 0.2)
        r = None if res_type is None else _rand((N, d), res_type, 3)
        mask = (torch.rand(N, device="cuda", generator=torch.Generator("cuda").manual_seed(4)) < 0.6).to(torch.uint8)
        _check_forward(mrl, x, w, r, None, out, block)
        _check_forward(mrl, x, w, r, mask, out, block)


@pytest.mark.parametrize("N", [1, 2, 3, 4, 5, 255, 256, 1023, 1024, 1025, 4097])
def test_forward_rows(mrl, N):
    """Counts of rows where the kernels change and workgroups end within their rows."""
    d = 1536
    x, w, r = _rand((4097, d), BF16, 1), 1 + _rand((d,), F32, 2, 0.2), _rand((4097, d), F32, 3)
    y, h, s = _check_forward(mrl, x[:N], w, r[:N], out=E4M3)
    one = mrl.rms_norm(x[N - 1:N], w, EPS, r[N - 1:N], out_dtype=E4M3)
    assert torch.equal(one[1], h[N - 1:])


def test_masked_rows_are_not_read(mrl):
    """NaN and infinities behind the mask leave no trace, in either pass; rows that the mask leaves empty altogether."""
    for N, d in ((9, 700), (2000, 257), (5, 6000)):
        for share in (0.0, 0.5):
            mask = (torch.arange(N, device="cuda") % 2 < 2 * share).to(torch.uint8)
            x, r, dy, w = _rand((N, d), BF16, 1), _rand((N, d), BF16, 2), _rand((N, d), BF16, 3), 1 + _rand((d,), BF16, 4, 0.2)
            res = _rand((N, d), BF16, 5)
            off = mask == 0
            bad = x.clone()
            bad[off] = float("nan")
            worse = dy.clone()
            worse[off] = float("inf")
            for out in (BF16, F32, E4M3):
                y, h, s = mrl.rms_norm(bad, w, EPS, r.masked_fill(off[:, None], float("inf")), mask, out)
                y0, h0, s0 = mrl.rms_norm(x, w, EPS, r, mask, out)
                assert torch.equal(y.float(), y0.float()) and torch.equal(h, h0) and bool((y[off].float() == 0).all()) and bool((h[off] == 0).all())
                assert s is None or torch.equal(s, s0)
            _check_forward(mrl, x, w, r, mask)
            for d_res in (None, res):
                dx, dw = mrl.rms_norm_backward(worse, bad, w, EPS, d_res, mask)
                dx0, dw0 = mrl.rms_norm_backward(dy, x, w, EPS, d_res, mask)
                assert torch.equal(dx, dx0) and torch.equal(dw, dw0)
                assert torch.equal(dx[off], (torch.zeros_like(res) if d_res is None else res)[off])
                if share == 0:
                    assert bool((dw == 0).all())


def test_rows_that_are_no_numbers(mrl):
    """Zero rows, infinities and NaN stay in their rows, and an 8-bit row says so in its scale."""
    N, d = 6, 300
    w = 1 + _rand((d,), F32, 1, 0.1)
    for t in (BF16, F32):
        x = _rand((N, d), t, 2)
        clean, _, clean_s = mrl.rms_norm(x, w, EPS, out_dtype=E4M3)
        x[1] = 0.0
        x[2, 17] = float("nan")
        x[3, 299] = float("inf")
        y, _, _ = mrl.rms_norm(x, w, EPS, out_dtype=F32)
        want = x.double() * torch.rsqrt(x.double().square().mean(1, keepdim=True) + EPS) * w.double()
        assert bool((y[1] == 0).all()) and bool(y[2].isnan().all())
        assert torch.equal(y.isnan(), want.float().isnan())
        q, _, s = mrl.rms_norm(x, w, EPS, out_dtype=E4M3)
        assert bool((q[1].float() == 0).all()) and float(s[1]) == np.float32(2.0 ** -100) / np.float32(448)
        assert bool(s[2].isnan()) and bool(q[2].float().isnan().all()) and bool(s[3].isnan())
        for n in (0, 4, 5):
            assert torch.equal(q[n].view(torch.uint8), clean[n].view(torch.uint8)) and s[n] == clean_s[n]
    # a weight that is infinite, and one that is NaN, in one block of 128 columns only
    x = _rand((2, d), F32, 3)
    for odd in (float("inf"), float("nan")):
        w2 = w.clone()
        w2[130] = odd
        q, _, s = mrl.rms_norm(x, w2, EPS, out_dtype=E4M3, scale_block=128)
        q0, _, s0 = mrl.rms_norm(x, w, EPS, out_dtype=E4M3, scale_block=128)
        assert bool((~s[:, 1].isfinite()).all()) and torch.equal(s[:, [0, 2]], s0[:, [0, 2]])
        keep = [*range(128), *range(256, d)]
        assert torch.equal(q.view(torch.uint8)[:, keep], q0.view(torch.uint8)[:, keep])


def test_magnitudes(mrl):
    """From the smallest rows that matter beside eps to ones whose mean square is near the largest float."""
    N, d = 8, 700
    scale = torch.tensor([1e-20, 1e-8, 1e-4, 1.0, 1e4, 1e9, 1e15, 1e17], device="cuda")[:, None]
    x = _rand((N, d), F32, 1) * scale
    w = 1 + _rand((d,), F32, 2, 0.2)
    _check_forward(mrl, x, w, out=F32)
    _check_forward(mrl, x, w, out=E4M3)
    dy = _rand((N, d), F32, 3)
    _check_backward(mrl, dy, x, w, dx_type=F32)


def _check_backward(mrl, dy, h, w, d_res=None, mask=None, dx_type=None, dw0=None, **kw):
    given = None if dw0 is None else dw0.clone()
    dx, dw = mrl.rms_norm_backward(dy, h, w, EPS, d_res, mask, dx_type, given, accumulate=given is not None, **kw)
    torch.cuda.synchronize()
    want_dx, want_dw, size_dx, size_dw = uo.rms_norm_backward(f64(dy), f64(h), f64(w), EPS, None if d_res is None else f64(d_res),
                                                              None if mask is None else mask.cpu().numpy())
    assert dx.dtype == (dx_type or h.dtype) and dw.dtype == F32
    # the two sums are off by 90 U of their absolute terms, r by 50 U; what they enter is measured by the size of dx's terms
    _within("dx", dx, want_dx, HALF[dx.dtype] * np.abs(want_dx) + 160 * U * size_dx + (1e-38 if dx.dtype == BF16 else 0))
    if dw0 is not None:
        want_dw, size_dw = want_dw + f64(dw0), size_dw + np.abs(f64(dw0))
        assert dw.data_ptr() == given.data_ptr()
    # a register adds the rows of its workgroup, one in 1024 at least; u itself is off by 52 U
    rows = -(-h.shape[0] // 1024) + 4
    _within("dweight", dw, want_dw, (56 + rows) * U * size_dw)
    return dx, dw


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("N", [1, 6])
def test_backward_widths(mrl, N, d):
    dy, h, w = _rand((N, d), BF16, d, 0.01), _rand((N, d), BF16, d + 1), 1 + _rand((d,), BF16, d + 2, 0.2)
    _check_backward(mrl, dy, h, w, _rand((N, d), BF16, d + 3, 0.01))
    _check_backward(mrl, dy.float(), h.float(), w.float(), dw0=_rand((d,), F32, d + 4))


@pytest.mark.parametrize("h_type", [BF16, F32])
@pytest.mark.parametrize("dy_type", [BF16, F32])
@pytest.mark.parametrize("dx_type", [BF16, F32])
@pytest.mark.parametrize("w_type", [BF16, F32])
def test_backward_types(mrl, h_type, dy_type, dx_type, w_type):
    for N, d in ((1500, 333), (3, 1000), (1030, 1800), (70, 5000), (3, 9000)):
        dy, h, w = _rand((N, d), dy_type, 1, 0.01), _rand((N, d), h_type, 2), 1 + _rand((d,), w_type, 3, 0.2)
        mask = (torch.rand(N, device="cuda", generator=torch.Generator("cuda").manual_seed(4)) < 0.6).to(torch.uint8)
        _check_backward(mrl, dy, h, w, None, None, dx_type)
        _check_backward(mrl, dy, h, w, _rand((N, d), h_type, 5, 0.01), mask, dx_type, dw0=_rand((d,), F32, 6))


@pytest.mark.parametrize("N", [2, 3, 4, 5, 1023, 1024, 1025, 4096, 4097, 9001])
@pytest.mark.parametrize("d", [64, 640, 1100])
def test_backward_rows(mrl, N, d):
    dy, h, w = _rand((N, d), BF16, 1, 0.01), _rand((N, d), BF16, 2), 1 + _rand((d,), F32, 3, 0.2)
    dx, dw = _check_backward(mrl, dy, h, w)
    again = mrl.rms_norm_backward(dy, h, w, EPS)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])           # bit-reproducible
    only, none = mrl.rms_norm_backward(dy, h, w, EPS, want_dweight=False)
    assert none is None and torch.equal(only, dx)


def test_gradient_against_differences(mrl):
    """Central differences of the forward pass itself, in 32 bits, along random directions: with y known to 1e-6 and steps of 1e-2
    the difference quotient of a sum of 400 terms is good to 1e-3 of the terms' size (second-order error 1e-4, rounding 1e-4)."""
    N, d = 5, 77
    x, r, w = _rand((N, d), F32, 1), _rand((N, d), F32, 2), 1 + _rand((d,), F32, 3, 0.2)
    dy, dh = _rand((N, d), F32, 4), _rand((N, d), F32, 5)

    def value(x, r, w):
        y, h, _ = mrl.rms_norm(x, w, EPS, r)
        return float((y.double() * dy.double()).sum() + (h.double() * dh.double()).sum())
    _, h, _ = mrl.rms_norm(x, w, EPS, r)
    dx, dw = mrl.rms_norm_backward(dy, h, w, EPS, d_residual=dh)
    for seed in range(3):
        for k, grad in ((0, dx), (1, dx), (2, dw)):
            at = [x, r, w]
            step = 1e-2 * _rand(at[k].shape, F32, 10 + seed)
            up, down = list(at), list(at)
            up[k], down[k] = at[k] + step, at[k] - step
            got = float((grad.double() * step.double()).sum())
            assert abs((value(*up) - value(*down)) / 2 - got) <= 1e-3 * float((grad.double() * step.double()).norm() * np.sqrt(step.numel())), (seed, k)


def test_slices_at_any_address(mrl):
    """Rows of odd widths that begin at any element of a larger buffer, and what lies in front of and behind the outputs."""
    for d, off in ((33, 1), (64, 3), (1537, 5), (513, 7)):
        N = 11
        big = _rand((N * d + 16,), BF16, d)
        x = big[off:off + N * d].view(N, d)
        w = _rand((d + 8,), BF16, 1)[off:off + d]
        assert x.is_contiguous() and x.data_ptr() % 16 != 0
        y, h, s = mrl.rms_norm(x, w, EPS, residual=x, out_dtype=E4M3)
        y2, h2, s2 = mrl.rms_norm(x.clone(), w.clone(), EPS, residual=x.clone(), out_dtype=E4M3)
        assert torch.equal(y.view(torch.uint8), y2.view(torch.uint8)) and torch.equal(h, h2) and torch.equal(s, s2)
        dx, dw = mrl.rms_norm_backward(x, x, w, EPS)
        dx2, dw2 = mrl.rms_norm_backward(x.clone(), x.clone(), w.clone(), EPS)
        assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
        # outputs inside guarded buffers, through the C interface
        for yt, code in ((BF16, 1), (F32, 0), (E4M3, 2)):
            guard = torch.full((N * d + 64,), 7.0, device="cuda").to(yt)
            sums = torch.full((N * d + 64,), 7.0, device="cuda", dtype=BF16)
            scales = torch.full((N + 2,), 7.0, device="cuda")
            item = guard.element_size()
            rc = mrl.lib().mrl_rms_norm(x.data_ptr(), x.data_ptr(), w.data_ptr(), None, N, d, EPS, 1, 1, 1, code, 0, sums.data_ptr() + 2 * off,
                                        guard.data_ptr() + item * off, scales.data_ptr() + 4 if code == 2 else None, None)
            torch.cuda.synchronize()
            assert rc == 0
            out = guard.float()
            assert bool((out[:off] == 7).all()) and bool((out[off + N * d:] == 7).all()) and torch.equal(sums[off:off + N * d].view(N, d), h)
            assert bool((sums[:off] == 7).all()) and bool((sums[off + N * d:] == 7).all())
            assert scales[0] == 7 and scales[-1] == 7
            if code == 2:
                assert torch.equal(out[off:off + N * d].view(N, d), y.float())
        guard = torch.full((N * d + 64,), 7.0, device="cuda", dtype=BF16)
        gw = torch.full((d + 2,), 7.0, device="cuda")
        ws = torch.empty(mrl.lib().mrl_rms_norm_backward_workspace(N, d), dtype=torch.uint8, device="cuda")
        rc = mrl.lib().mrl_rms_norm_backward(x.data_ptr(), x.data_ptr(), w.data_ptr(), None, None, N, d, EPS, 1, 1, 1, 1, 0, guard.data_ptr() + 2 * off,
                                             gw.data_ptr() + 4, ws.data_ptr(), ws.numel(), None)
        torch.cuda.synchronize()
        assert rc == 0 and torch.equal(guard[off:off + N * d].view(N, d), dx) and torch.equal(gw[1:-1], dw)
        assert bool((guard[:off] == 7).all()) and bool((guard[off + N * d:] == 7).all()) and gw[0] == 7 and gw[-1] == 7


@pytest.mark.parametrize("N,d", [(3, 100), (700, 9), (50, 1001), (1200, 1536), (700, 1537), (300, 4099), (2, 9000), (20, 12345)])
def test_outputs_in_the_inputs_buffers(mrl, N, d):
    x, r, w = _rand((N, d), BF16, 1), _rand((N, d), BF16, 2), _rand((d,), BF16, 3)
    y, h, _ = mrl.rms_norm(x, w, EPS, r)
    x2, r2 = x.clone(), r.clone()
    assert mrl.lib().mrl_rms_norm(x2.data_ptr(), r2.data_ptr(), w.data_ptr(), None, N, d, EPS, 1, 1, 1, 1, 0, r2.data_ptr(), x2.data_ptr(), None, None) == 0
    assert torch.equal(x2, y) and torch.equal(r2, h)
    dx, dw = mrl.rms_norm_backward(x, h, w, EPS, d_residual=r)
    for k in range(3):
        t = [x.clone(), h.clone(), r.clone()]
        assert mrl.lib().mrl_rms_norm_backward(t[0].data_ptr(), t[1].data_ptr(), w.data_ptr(), t[2].data_ptr(), None, N, d, EPS, 1, 1, 1, 1, 0,
                                               t[k].data_ptr(), None, None, 0, None) == 0
        assert torch.equal(t[k], dx)


def test_more_than_2_31_elements(mrl):
    """Rows whose elements lie beyond the largest 32-bit signed offset."""
    d = 4100
    N = 2 ** 31 // d + 500
    x = torch.zeros((N, d), device="cuda", dtype=BF16)
    tail = _rand((300, d), BF16, 1)
    x[-300:] = tail
    w = 1 + _rand((d,), F32, 2, 0.2)
    mask = torch.zeros(N, dtype=torch.uint8, device="cuda")
    mask[-300:] = 1
    mask[0] = 1
    y, h, s = mrl.rms_norm(x, w, EPS, residual=x, token_mask=mask, out_dtype=E4M3)
    y0, h0, s0 = mrl.rms_norm(tail, w, EPS, residual=tail, out_dtype=E4M3)
    assert torch.equal(h[-300:], h0) and bool((h[:1000] == 0).all())
    assert torch.equal(y[-300:].float(), y0.float()) and torch.equal(s[-300:], s0)
    del y, h
    dx, dw = mrl.rms_norm_backward(x, x, w, EPS, token_mask=mask)
    dx0, dw0 = mrl.rms_norm_backward(tail, tail, w, EPS)
    assert torch.equal(dx[-300:], dx0) and torch.allclose(dw, dw0, rtol=1e-5, atol=1e-4)


@pytest.mark.parametrize("N,d", [(2 ** 21 + 77, 264), (2 ** 25 + 4097, 9)])
def test_more_rows_than_a_launch_is_wide(mrl, N, d):
    """More workgroups than go along x; rows of few columns, several to a wave, among them."""
    x = torch.zeros((N, d), device="cuda", dtype=BF16)
    head, tail = _rand((100, d), BF16, 1), _rand((300, d), BF16, 2)
    x[:100], x[-300:] = head, tail
    w = 1 + _rand((d,), F32, 3, 0.2)
    y, _, _ = mrl.rms_norm(x, w, EPS)
    assert torch.equal(y[:100], mrl.rms_norm(head, w, EPS)[0]) and torch.equal(y[-300:], mrl.rms_norm(tail, w, EPS)[0])
    assert not bool(y[100:-300].any())
    dx, dw = mrl.rms_norm_backward(x, x, w, EPS)
    ends = torch.cat([head, tail])
    dx0, dw0 = mrl.rms_norm_backward(ends, ends, w, EPS)
    assert torch.equal(dx[:100], dx0[:100]) and torch.equal(dx[-300:], dx0[100:])
    # zeros beside them change no sum, only its order: 4 + 400 additions
    assert torch.all((dw - dw0).abs() <= 404 * U * (ends.double().square() / (ends.double().square().mean(1, keepdim=True) + EPS).sqrt()).sum(0))


def test_mask_in_the_shape_of_the_batch(mrl):
    """A mask [B, T] serves the rows [B * T, d], as it does the scoring step."""
    B, T, d = 5, 37, 200
    x, w = _rand((B * T, d), BF16, 1), _rand((d,), BF16, 2)
    mask = (torch.arange(T, device="cuda")[None] < torch.tensor([0, 1, 17, 36, 37], device="cuda")[:, None]).to(torch.uint8)
    for a, b in zip(mrl.rms_norm(x, w, EPS, x, mask, E4M3), mrl.rms_norm(x, w, EPS, x, mask.reshape(-1), E4M3)):
        assert torch.equal(a.float(), b.float())
    _check_backward(mrl, x, x, w, None, mask.reshape(-1))
    for a, b in zip(mrl.rms_norm_backward(x, x, w, EPS, None, mask), mrl.rms_norm_backward(x, x, w, EPS, None, mask.reshape(-1))):
        assert torch.equal(a, b)


def test_no_rows(mrl):
    w = torch.ones(16, device="cuda")
    x = torch.empty((0, 16), device="cuda")
    y, h, s = mrl.rms_norm(x, w, EPS, residual=x, out_dtype=E4M3, scale_block=128)
    assert y.shape == (0, 16) and h.shape == (0, 16) and s.shape == (0, 1)
    dx, dw = mrl.rms_norm_backward(x, x, w, EPS)
    assert dx.shape == (0, 16) and bool((dw == 0).all())
    kept = torch.full((16,), 3.0, device="cuda")
    _, dw = mrl.rms_norm_backward(x, x, w, EPS, out_dweight=kept, accumulate=True)
    assert bool((dw == 3).all())


def test_another_device_is_refused(mrl, monkeypatch):
    """Tensors that are not on the current device, whose stream the call would use."""
    from paper_2605_07244_amd import binding
    x, w = _rand((4, 16), BF16, 1), torch.ones(16, device="cuda")
    p, g = torch.zeros(10, device="cuda"), torch.zeros(10, device="cuda")
    plan = mrl.adamw_plan([p], [g])
    monkeypatch.setattr(binding, "_native", False)
    monkeypatch.setattr(binding.torch.cuda, "current_device", lambda: 1)
    for call in (lambda: mrl.rms_norm(x, w), lambda: mrl.rms_norm_backward(x, x, w), lambda: mrl.grad_norm(plan, 1.0), lambda: mrl.adamw_step(plan, 1e-3, 1),
                 lambda: mrl.grad_plan([g])):
        with pytest.raises(ValueError, match="current device"):
            call()


def test_refusals(mrl):
    x, w = torch.zeros((4, 16), device="cuda"), torch.ones(16, device="cuda")
    for bad in (lambda: mrl.rms_norm(x.t(), torch.ones(4, device="cuda")), lambda: mrl.rms_norm(x[:, ::2], w[::2]),
                lambda: mrl.rms_norm(x, w, residual=x[:3]), lambda: mrl.rms_norm(x, w, token_mask=torch.ones(5, dtype=torch.uint8, device="cuda")),
                lambda: mrl.rms_norm_backward(x, x, w, out_dweight=torch.ones(17, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: mrl.rms_norm(x.half(), w), lambda: mrl.rms_norm(x, w.half()), lambda: mrl.rms_norm(x, w, residual=x.half()),
                lambda: mrl.rms_norm(x, w, token_mask=torch.ones(4, device="cuda")), lambda: mrl.rms_norm(x, w.cpu()),
                lambda: mrl.rms_norm_backward(x, x, w, out_dweight=w.bfloat16()), lambda: mrl.rms_norm(x, w, out_dtype=torch.int8)):
        with pytest.raises(TypeError):
            bad()
    for bad, status in ((lambda: mrl.rms_norm(x, w, eps=0.0), -7), (lambda: mrl.rms_norm(x, w, scale_block=128), -7),
                        (lambda: mrl.rms_norm(x, w, out_dtype=E4M3, scale_block=64), -7), (lambda: mrl.rms_norm(x.bfloat16(), w, out_dtype=E4M3, scale_block=-1), -7),
                        (lambda: mrl.rms_norm(torch.zeros((1, 16385), device="cuda"), torch.ones(16385, device="cuda")), -2),
                        (lambda: mrl.rms_norm(x, w, residual=x.bfloat16()), -3),
                        (lambda: mrl.rms_norm_backward(x, x, w, eps=-1.0), -7),
                        (lambda: mrl.rms_norm_backward(x, x, w, workspace=torch.empty(256, dtype=torch.uint8, device="cuda")[:16]), -6)):
        with pytest.raises(mrl.MrlError) as e:
            bad()
        assert e.value.status == status


def test_both_ways_of_marshalling(mrl, monkeypatch):
    """The extension and ctypes give the same results."""
    from paper_2605_07244_amd import binding
    N, d = 70, 300
    x, r, w, dy = _rand((N, d), BF16, 1), _rand((N, d), F32, 2), _rand((d,), F32, 3), _rand((N, d), F32, 4)
    mask = (torch.arange(N, device="cuda") % 3 > 0).to(torch.uint8)

    def results():
        out = []
        for t, block in ((F32, 0), (BF16, 0), (E4M3, 0), (E4M3, 128)):
            out += list(mrl.rms_norm(x, w, EPS, r, mask, t, block)) + list(mrl.rms_norm(x, w, EPS, out_dtype=t, scale_block=block))
        out += list(mrl.rms_norm_backward(dy, r, w, EPS, r, mask, BF16))
        out += list(mrl.rms_norm_backward(dy, x, w, EPS, None, None, None, torch.ones(d, device="cuda"), True))
        out += list(mrl.rms_norm_backward(dy, x, w, EPS, want_dweight=False))
        return out
    fast = results()
    monkeypatch.setattr(binding, "_HOST", binding._NoHost)
    slow = results()
    assert len(fast) == len(slow)
    for a, b in zip(fast, slow):
        assert (a is None) == (b is None)
        if a is not None:
            assert a.dtype == b.dtype and a.shape == b.shape and torch.equal(a.float(), b.float())


def test_on_another_stream(mrl):
    """The calls run on the current stream: results of a chain on a side stream, with the default stream busy."""
    N, d = 3000, 2048
    x, w, dy = _rand((N, d), BF16, 1), 1 + _rand((d,), F32, 2, 0.2), _rand((N, d), BF16, 3)
    y0, h0, _ = mrl.rms_norm(x, w, EPS, x)
    dx0, dw0 = mrl.rms_norm_backward(dy, h0, w, EPS)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    busy = torch.randn((4096, 4096), device="cuda")
    for _ in range(3):
        busy = busy @ busy * 1e-3
    with torch.cuda.stream(side):
        x2 = x * 1                                       # produced on the side stream
        y, h, _ = mrl.rms_norm(x2, w, EPS, x2)
        dx, dw = mrl.rms_norm_backward(dy, h, w, EPS)
    side.synchronize()
    assert torch.equal(y, y0) and torch.equal(dx, dx0) and torch.equal(dw, dw0)


def test_captured_and_replayed(mrl):
    N, d = 300, 1536
    x, r, w, dy = _rand((N, d), BF16, 1), _rand((N, d), BF16, 2), 1 + _rand((d,), F32, 3, 0.2), _rand((N, d), BF16, 4)
    dw = torch.zeros(d, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        mrl.rms_norm(x, w, EPS, r)
        mrl.rms_norm_backward(dy, r, w, EPS)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, h, _ = mrl.rms_norm(x, w, EPS, r)
        q, _, s = mrl.rms_norm(x, w, EPS, r, out_dtype=E4M3)
        dx, _ = mrl.rms_norm_backward(dy, h, w, EPS, out_dweight=dw, accumulate=True)
    total = torch.zeros(d, device="cuda")
    for k in range(4):
        x.copy_(_rand((N, d), BF16, 10 + k))
        dy.copy_(_rand((N, d), BF16, 20 + k))
        graph.replay()
        torch.cuda.synchronize()
        y1, h1, _ = mrl.rms_norm(x, w, EPS, r)
        q1, _, s1 = mrl.rms_norm(x, w, EPS, r, out_dtype=E4M3)
        dx1, _ = mrl.rms_norm_backward(dy, h1, w, EPS, out_dweight=total, accumulate=True)
        assert torch.equal(y, y1) and torch.equal(h, h1) and torch.equal(q.float(), q1.float()) and torch.equal(s, s1)
        assert torch.equal(dx, dx1) and torch.equal(dw, total), k


def test_no_rows_without_a_weight_gradient(mrl):
    w = torch.ones(16, device="cuda")
    for x_type in (F32, BF16):
        x = torch.empty((0, 16), device="cuda", dtype=x_type)
        for mask in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
            dx, dw = mrl.rms_norm_backward(x, x, w, EPS, x, mask, want_dweight=False)
            assert dx.shape == (0, 16) and dx.dtype == x_type and dw is None


def test_masked_gradient_against_differences(mrl):
    """Differences of the forward pass, with its bound in test_gradient_against_differences: without a mask where only some rows' y are used, and of two masked
    norms, one behind the other along the residual stream."""
    N, d = 7, 77
    x, r, b = (_rand((N, d), F32, k) for k in (1, 2, 3))
    w, w2 = 1 + _rand((d,), F32, 4, 0.2), 1 + _rand((d,), F32, 5, 0.2)
    dy, dh = _rand((N, d), F32, 6), _rand((N, d), F32, 7)
    mask = (torch.arange(N, device="cuda") % 3 != 1).to(torch.uint8)
    on = mask.double()[:, None]

    def unmasked(x, r, w):
        y, h, _ = mrl.rms_norm(x, w, EPS, r)
        return float((y.double() * dy.double() * on).sum() + (h.double() * dh.double()).sum())

    def masked(x, r, w):
        y, h, _ = mrl.rms_norm(x, w, EPS, r, mask)
        y2, _, _ = mrl.rms_norm(b, w2, EPS, h, mask)
        return float((y.double() * dy.double()).sum() + (y2.double() * dh.double()).sum())
    _, h, _ = mrl.rms_norm(x, w, EPS, r)
    one = mrl.rms_norm_backward(dy, h, w, EPS, dh, mask)
    _, h, _ = mrl.rms_norm(x, w, EPS, r, mask)
    _, h2, _ = mrl.rms_norm(b, w2, EPS, h, mask)
    back, _ = mrl.rms_norm_backward(dh, h2, w2, EPS, None, mask)
    two = mrl.rms_norm_backward(dy, h, w, EPS, back, mask)
    assert not bool(back[mask == 0].any()) and not bool(two[0][mask == 0].any())
    for value, (dx, dw) in ((unmasked, one), (masked, two)):
        for seed in range(3):
            for k, grad in ((0, dx), (1, dx), (2, dw)):
                at = [x, r, w]
                step = 1e-2 * _rand(at[k].shape, F32, 10 + seed)
                up, down = list(at), list(at)
                up[k], down[k] = at[k] + step, at[k] - step
                got = float((grad.double() * step.double()).sum())
                assert abs((value(*up) - value(*down)) / 2 - got) <= 1e-3 * float((grad.double() * step.double()).norm() * np.sqrt(step.numel())), (value, seed, k)


@pytest.mark.parametrize("d", [128, 1536, 2048, 3584])
@pytest.mark.parametrize("N", [16384, 20001])
@pytest.mark.parametrize("types", [(BF16, BF16, BF16), (F32, F32, F32)])
def test_backward_of_long_calls(mrl, N, d, types):
    """Calls long enough for the most workgroups, with data in every row, against 64 bits (on the GPU): with and without d_residual, which are other counts
    of workgroups, every row scored, and sequences of 512 slots with scored heads, a period that divides those counts.

    A workgroup's register adds its rows one after the other.  The workspace holds a row of partial sums for each workgroup of a call without
    d_residual; with one there are at least half as many.  Then at most 6 additions join lanes and waves, the rest is fp64 and one rounding; u is off by 52 U."""
    h_type, dy_type, w_type = types
    dy, h, w = _rand((N, d), dy_type, 1, 0.01), _rand((N, d), h_type, 2, 2.0), 1 + _rand((d,), w_type, 3, 0.2)
    res = _rand((N, d), h_type, 4, 0.01)
    lengths = torch.randint(0, 513, (N // 512 + 1, 1), device="cuda", generator=torch.Generator("cuda").manual_seed(5))
    heads = (torch.arange(512, device="cuda")[None] < lengths).to(torch.uint8).reshape(-1)[:N].contiguous()
    groups = mrl.lib().mrl_rms_norm_backward_workspace(N, d) // (4 * d)
    for d_res in (None, res):
        rows = -(-N // groups) * (1 if d_res is None else 2)
        for mask in (None, heads):
            dx, dw = mrl.rms_norm_backward(dy, h, w, EPS, d_res, mask)
            on = torch.ones(N, 1, device="cuda", dtype=torch.float64) if mask is None else mask.double()[:, None]
            h64, g64 = h.double() * on, dy.double() * on
            r = 1 / torch.sqrt((h64 * h64).mean(1, keepdim=True) + EPS)
            u, g = h64 * r, g64 * w.double()
            want = r * (g - u * (g * u).mean(1, keepdim=True))
            size = r * (g.abs() + u.abs() * (g * u).abs().mean(1, keepdim=True))
            if d_res is not None:
                want, size = want + d_res.double(), size + d_res.double().abs()
            bound = HALF[h_type] * want.abs() + 160 * U * size + 1e-38
            assert bool(((dx.double() - want).abs() <= bound).all()), (d_res is None, mask is None)
            err, bound = (dw.double() - (g64 * u).sum(0)).abs(), (52 + rows + 6 + 1) * U * (g64 * u).abs().sum(0)
            print("dweight: worst error over its bound", float((err / bound).max()))
            assert bool((err <= bound).all()), (d_res is None, mask is None)
            again = mrl.rms_norm_backward(dy, h, w, EPS, d_res, mask)
            assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])


def test_codes_differ_at_borders_only(mrl):
    """8-bit codes are those of the exact quotient, but where it lies at the border of two of them: y is off by 52 U, the scale by 54 U and the quotient by
    2 roundings.  They are the same bits again in outputs that hold something else before."""
    for N, d, block in ((2047, 3584, 0), (1000, 700, 128)):
        x, r, w = _rand((N, d), BF16, 1), _rand((N, d), BF16, 2, 3.0), 1 + _rand((d,), BF16, 3, 0.2)
        y, h, s = mrl.rms_norm(x, w, EPS, r, out_dtype=E4M3, scale_block=block)
        for fill in (0x55, 0xFF):
            junk = [torch.full((N * d * size,), fill, dtype=torch.uint8, device="cuda") for size in (1, 2)]
            del junk
            again = mrl.rms_norm(x, w, EPS, r, out_dtype=E4M3, scale_block=block)
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip((y, h, s), again))
        h64 = x.double() + r.double()
        y64 = h64 / torch.sqrt((h64 * h64).mean(1, keepdim=True) + EPS) * w.double()
        scale = torch.stack([part.abs().amax(1) for part in y64.split(block or d, dim=1)], dim=1) / 448
        z = (y64 / scale.repeat_interleave(block or d, dim=1)[:, :d]).abs()
        step = torch.exp2(torch.floor(torch.log2(z.clamp(min=2.0 ** -6))) - 3)
        want = torch.round(z / step) * step * torch.sign(y64)
        other = y.double() != want
        border = (torch.abs(torch.frac(z / step) - 0.5) * step)[other]
        print("codes off the exact ones:", int(other.sum()), "of", N * d)
        assert bool((border <= 108 * U * z[other]).all())
        assert bool(((y.double() - want).abs() <= step)[other].all())
