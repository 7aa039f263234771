"""Norm, gradient norm and AdamW: refusals of the C ABI and of the binding, and the rounding of 8-bit moments, without a GPU."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2605_07244_amd as m
from paper_2605_07244_amd import binding
from tests import update_oracle as uo

P = ctypes.c_void_p
FAKE = P(0x1000)                       # never dereferenced: validation fails first
NO_GPU = (-8, -9)                      # where every argument is right, the call ends at the device check


def _gpu():
    return torch.cuda.is_available()


def _norm(x=FAKE, res=None, w=FAKE, mask=None, N=4, d=64, eps=1e-6, xt=1, rt=1, wt=1, yt=1, block=0, h=None, y=FAKE, scale=None):
    return m.lib().mrl_rms_norm(x, res, w, mask, N, d, eps, xt, rt, wt, yt, block, h, y, scale, None)


def test_rms_norm_argument_errors():
    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(res=FAKE), dict(h=FAKE), dict(yt=2), dict(scale=FAKE)):
        assert _norm(**bad) == -1, bad
    for bad in (dict(N=-1), dict(N=(1 << 30) + 1), dict(d=0), dict(d=-3), dict(d=16385)):
        assert _norm(**bad) == -2, bad
    for bad in (dict(xt=2), dict(xt=7), dict(wt=2), dict(yt=3), dict(yt=-1), dict(xt=0, res=FAKE, rt=1, h=FAKE), dict(res=FAKE, rt=2, h=FAKE)):
        assert _norm(**bad) == -3, bad
    for bad in (dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(block=128), dict(block=64, yt=2, scale=FAKE),
                dict(block=-128, yt=2, scale=FAKE)):
        assert _norm(**bad) == -7, bad
    assert _norm(N=0, x=None, w=None, y=None) == 0
    if not _gpu():
        assert _norm() in NO_GPU and _norm(yt=2, scale=FAKE, block=128) in NO_GPU and _norm(res=FAKE, rt=0, h=FAKE) in NO_GPU


def _back(dy=FAKE, h=FAKE, w=FAKE, res=None, mask=None, N=4, d=64, eps=1e-6, types=(1, 1, 1, 1), acc=0, dx=FAKE, dw=FAKE, ws=FAKE, ws_bytes=1 << 30):
    return m.lib().mrl_rms_norm_backward(dy, h, w, res, mask, N, d, eps, *types, acc, dx, dw, ws, ws_bytes, None)


def test_rms_norm_backward_argument_errors():
    for bad in (dict(dy=None), dict(h=None), dict(w=None), dict(dx=None)):
        assert _back(**bad) == -1, bad
    for bad in (dict(N=-1), dict(d=0), dict(d=16385)):
        assert _back(**bad) == -2, bad
    for k in range(4):
        assert _back(types=[2 if i == k else 1 for i in range(4)]) == -3
    for bad in (dict(eps=0.0), dict(eps=float("nan")), dict(acc=2), dict(acc=-1)):
        assert _back(**bad) == -7, bad
    need = m.lib().mrl_rms_norm_backward_workspace(4, 64)
    assert need > 0 and need % 256 == 0
    for bad in (dict(ws=None), dict(ws=P(0x1001)), dict(ws_bytes=need - 1)):
        assert _back(**bad) == -6, bad
    assert _back(N=0, acc=1) == 0 and _back(N=0, dw=None) == 0
    for N, d in ((-1, 64), (4, 0), (4, 16385)):
        assert m.lib().mrl_rms_norm_backward_workspace(N, d) == 0
    if not _gpu():
        assert _back() in NO_GPU and _back(dw=None, ws=None, ws_bytes=0) in NO_GPU


def _tensors(*rows):
    table = (binding._ParamTensor * len(rows))()
    for t, row in zip(table, rows):
        t.param, t.grad, t.m, t.v, t.n = 0x10000, 0x20000, 0x30000, 0x40000, 100
        for k, v in row.items():
            setattr(t, k, v)
    return table


def test_grad_norm_argument_errors():
    L = m.lib()
    t = _tensors({})
    need = L.mrl_grad_norm_workspace(t, 1)
    f = lambda t=t, n=1, most=1.0, out=FAKE, ws=FAKE, size=1 << 20: L.mrl_grad_norm(t, n, most, out, ws, size, None)
    assert f(out=None) == -1 and f(t=None) == -1 and f(t=_tensors(dict(grad=None))) == -1
    assert f(n=-1) == -2 and f(t=_tensors(dict(n=-1))) == -2 and f(t=_tensors(dict(n=(1 << 40) + 1))) == -2
    assert f(t=_tensors(dict(grad_dtype=2))) == -3
    for most in (0.0, -1.0, float("nan")):
        assert f(most=most) == -7
    assert f(ws=None) == -6 and f(ws=P(0x1001)) == -6 and f(size=need - 1) == -6
    assert L.mrl_grad_norm_workspace(_tensors(dict(n=-1)), 1) == 0
    # tensors that together pass the count of workgroups of a launch
    assert f(t=_tensors(*[dict(n=1 << 40)] * 5), n=5) == -2
    if not _gpu():
        assert f() in NO_GPU and f(n=0, t=None) in NO_GPU


def _step(rows=({},), count=None, coef=None, **kw):
    c = binding._AdamWConfig(1e-3, 0.9, 0.999, 1e-8, 1, 0, 0, 0, None, None)
    for k, v in kw.items():
        setattr(c, k, v)
    t = _tensors(*rows)
    return m.lib().mrl_adamw(t, len(rows) if count is None else count, ctypes.byref(c), coef, None)


def test_adamw_argument_errors():
    assert m.lib().mrl_adamw(_tensors({}), 1, None, None, None) == -1
    for row in (dict(param=None), dict(grad=None), dict(m=None), dict(v=None)):
        assert _step([row]) == -1, row
    assert _step([{}], state_dtype=2) == -1                           # 8-bit moments need their scales
    assert _step(count=-1) == -2 and _step([dict(n=-1)]) == -2
    assert _step(state_dtype=1) == -3 and _step([dict(grad_dtype=2)]) == -3
    nan, inf = float("nan"), float("inf")
    for kw in (dict(lr=-1.0), dict(lr=nan), dict(lr=inf), dict(beta1=1.0), dict(beta1=-0.1), dict(beta1=nan), dict(beta2=1.0), dict(beta2=nan),
               dict(eps=0.0), dict(eps=nan), dict(eps=-1.0), dict(step=0), dict(step=-5), dict(skip_nonfinite=2)):
        assert _step(**kw) == -7, kw
    for decay in (-0.1, nan, inf):
        assert _step([dict(weight_decay=decay)]) == -7
    assert _step([], count=0) == 0
    if not _gpu():
        assert _step() in NO_GPU and _step([dict(n=0, param=None, grad=None, m=None, v=None)]) in NO_GPU
        assert _step(step=0, step_dev=0x1000) in NO_GPU


def test_overlapping_buffers_are_found():
    check = lambda *rows, dtype=0: m.lib().mrl_adamw_check(_tensors(*rows), len(rows), dtype)
    apart = dict(param=0x110000, grad=0x120000, m=0x130000, v=0x140000)
    assert check({}) == 0 and check({}, apart) == 0
    assert check({}, {}) == -7                                        # the same tensor twice
    assert check({}, dict(apart, param=0x10000)) == -7
    assert check({}, dict(apart, v=0x30000 + 399)) == -7              # by a byte
    assert check({}, dict(apart, v=0x30000 + 400)) == 0               # one right behind the other
    assert check(dict(m=0x40000)) == -7 and check(dict(m=0x20000)) == -7
    assert check(dict(param=0x20000 + 396)) == -7                     # a gradient that is written to
    assert check({}, dict(apart, grad=0x20000 + 40)) == 0             # gradients may overlap
    assert check(dict(copy=0x10000)) == -7 and check(dict(copy=0x50000)) == 0
    codes = dict(m_scale=0x60000, v_scale=0x70000)
    assert check(codes, dtype=2) == 0 and check(dict(codes, v_scale=0x60000), dtype=2) == -7
    assert check(dict(codes, v=0x30000 + 100), dtype=2) == 0          # codes are a byte each
    assert check(dict(n=0, m=0x40000)) == 0 and check(dtype=1) == -3


def test_binding_refusals():
    """What the binding checks itself, before the library is asked."""
    x, w = torch.zeros(4, 8), torch.zeros(8)
    for bad in (dict(residual=torch.zeros(4, 7)), dict(token_mask=torch.zeros(3, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            m.rms_norm(x, w, **bad)
    with pytest.raises(ValueError):
        m.rms_norm(x[0], w)
    with pytest.raises(ValueError):
        m.rms_norm(x, w[:7])
    with pytest.raises(TypeError):
        m.rms_norm(x, w, out_dtype=torch.float16)
    with pytest.raises(TypeError):
        m.rms_norm(x.double(), w)
    with pytest.raises(TypeError, match="GPU"):
        m.rms_norm(x, w)
    for bad in (dict(d_residual=torch.zeros(3, 8)), dict(out_dweight=torch.zeros(9)), dict(accumulate=True)):
        with pytest.raises(ValueError):
            m.rms_norm_backward(x, x, w, **bad)
    with pytest.raises(TypeError):
        m.rms_norm_backward(x, x, w, d_residual=x.bfloat16())
    with pytest.raises(TypeError):
        m.rms_norm_backward(x, x, w, dx_dtype=torch.float64)
    with pytest.raises(TypeError, match="GPU"):
        m.rms_norm_backward(x, x, w)
    with pytest.raises(TypeError, match="GPU"):
        m.grad_plan([w])
    with pytest.raises(TypeError, match="GPU"):
        m.adamw_plan([w], [w])


def test_structures_match_the_header():
    assert ctypes.sizeof(binding._ParamTensor) == 72 and ctypes.sizeof(binding._AdamWConfig) == 72


def test_codes_of_the_oracle():
    """The values that the 8-bit oracle rounds to are the e4m3 values, and its roundings have the mean they should."""
    values = np.unique(np.abs(torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()))
    values = values[np.isfinite(values)].astype(np.float64)
    rng = np.random.default_rng(1)
    x = np.concatenate([values, np.exp(rng.uniform(np.log(1e-4), np.log(448), 4000))])
    lo = values[np.searchsorted(values, x, side="right") - 1]
    hi = values[np.minimum(np.searchsorted(values, x, side="left"), len(values) - 1)]
    assert np.array_equal(uo.to_code(x, np.zeros_like(x)), lo)
    assert np.array_equal(uo.to_code(x, np.full_like(x, 1 - 2.0 ** -40)), hi)
    n = 1 << 20
    bits = uo.random_bits(n, seed=77, step=3, place=2)
    for u in ((bits & 0xFFFF) / 65536.0, (bits >> 16) / 65536.0):
        # a uniform variable: mean 1/2 within 5 standard deviations, no two neighbours alike more often than chance has it
        assert abs(u.mean() - 0.5) < 5 * 0.2887 / np.sqrt(n)
        assert abs(np.corrcoef(u[:-1], u[1:])[0, 1]) < 5 / np.sqrt(n)
        share = np.bincount((u * 16).astype(int), minlength=16) / n
        assert np.all(np.abs(share - 1 / 16) < 5 * np.sqrt(1 / 16 * 15 / 16 / n))
    a, b = (bits & 0xFFFF) / 65536.0, (bits >> 16) / 65536.0
    assert abs(np.corrcoef(a, b)[0, 1]) < 5 / np.sqrt(n)
    for other in (dict(seed=78, step=3, place=2), dict(seed=77, step=4, place=2), dict(seed=77, step=3, place=3), dict(seed=77 + (1 << 32), step=3, place=2)):
        assert np.mean(uo.random_bits(n, **other) == bits) < 1e-3


def test_no_rows_need_no_pointers():
    """An empty tensor has no device pointer: a call of no rows that asks for no weight gradient has none at all."""
    for pointers in (dict(dx=None), dict(dx=None, dy=None, h=None, w=None, ws=None, ws_bytes=0)):
        assert _back(N=0, dw=None, **pointers) == 0, pointers
    assert _back(N=0, dw=None, dx=None, d=0) == -2 and _back(N=0, dw=None, dx=None, eps=0.0) == -7


def test_numbers_past_32_bits_are_refused(monkeypatch):
    """The C interface takes widths and scale blocks in 32 bits.  Cut to them, 2^32 + 128 would be a block of 128 next to an output with one scale a
    row, and a row of 2^32 + 16 columns one of 16.  (Tensors that are not on a GPU: these are checked before anything needs one.)"""
    x, w = torch.zeros(4, 256), torch.zeros(256)
    for block in ((1 << 32) + 128, 1 << 32, -(1 << 32), 1 << 31, 1 << 70):
        with pytest.raises(ValueError, match="scale_block"):
            m.rms_norm(x, w, out_dtype=torch.float8_e4m3fn, scale_block=block)
    for d in (1 << 31, (1 << 32) + 16):
        x, w = torch.empty((1, d), device="meta"), torch.empty(d, device="meta")
        with pytest.raises(ValueError, match="columns"):
            m.rms_norm(x, w)
        with pytest.raises(ValueError, match="columns"):
            m.rms_norm_backward(x, x, w)
    # a step is counted in 64 bits
    monkeypatch.setattr(binding, "_native", False)
    plan = object.__new__(m.AdamWPlan)
    for name, value in dict(address=0, count=0, workspace=torch.zeros(1, dtype=torch.uint8), state_dtype=binding.F32, table=None).items():
        setattr(plan, name, value)
    for step in (1 << 63, (1 << 64) + 5):
        with pytest.raises(ValueError, match="step"):
            m.adamw_step(plan, 1e-3, step)


def test_plans_of_no_tensors_are_refused():
    """A parameter without a gradient has None in its place; so have lists that do not hold what they should."""
    w = torch.zeros(8)
    for bad in (lambda: m.grad_plan([None]), lambda: m.grad_plan([w, None]), lambda: m.adamw_plan([w], [None]), lambda: m.grad_plan([1.0]),
                lambda: m.adamw_plan([w], [w], m=[None]), lambda: m.adamw_plan([w], [w], m=["m"])):
        with pytest.raises(TypeError, match="must hold tensors"):
            bad()


def _differences(value, x, step=1e-6):
    out = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += step
        down[i] -= step
        out[i] = (value(up) - value(down)) / (2 * step)
    return out


def test_masked_backward_and_the_forwards_it_belongs_to():
    """In 64 bits: steps of 1e-6 leave 1e-12 of third derivatives and 1e-16 / 1e-6 of rounding, both times the terms' size (10)."""
    rng = np.random.default_rng(1)
    N, d = 6, 5
    x, r, w, w2 = rng.normal(size=(N, d)), rng.normal(size=(N, d)), 1 + 0.2 * rng.normal(size=d), 1 + 0.2 * rng.normal(size=d)
    dy, dh, b = (rng.normal(size=(N, d)) for _ in range(3))
    mask = np.array([1, 0, 1, 1, 0, 1])

    # the residual stream runs through every row, the loss reads y of the scored ones
    def unmasked(x):
        y, h = uo.rms_norm(x, w, 1e-5, r)
        return np.sum((y * dy)[mask == 1]) + np.sum(h * dh)
    dx = uo.rms_norm_backward(dy, x + r, w, 1e-5, dh, mask)[0]
    assert np.max(np.abs(_differences(unmasked, x) - dx)) < 1e-8

    # two masked norms, the second one's residual stream the first one's h: the gradient that comes back along it is zero in the other rows
    def masked(x):
        y, h = uo.rms_norm(x, w, 1e-5, r, mask)
        y2, _ = uo.rms_norm(b, w2, 1e-5, h, mask)
        return np.sum(y * dy) + np.sum(y2 * dh)
    _, h = uo.rms_norm(x, w, 1e-5, r, mask)
    _, h2 = uo.rms_norm(b, w2, 1e-5, h, mask)
    back = uo.rms_norm_backward(dh, h2, w2, 1e-5, None, mask)[0]
    dx = uo.rms_norm_backward(dy, h, w, 1e-5, back, mask)[0]
    assert not back[mask == 0].any() and not dx[mask == 0].any()
    assert np.max(np.abs(_differences(masked, x) - dx)) < 1e-8
    # and one that does not come from such a call is not its gradient there, until it is cleared
    dx = uo.rms_norm_backward(dy, h, w, 1e-5, dh, mask)[0]
    want = _differences(lambda x: np.sum(uo.rms_norm(x, w, 1e-5, r, mask)[0] * dy) + np.sum(uo.rms_norm(x, w, 1e-5, r, mask)[1] * dh), x)
    assert np.array_equal((np.abs(want - dx) > 1e-8).any(axis=1), mask == 0)
    dx = uo.rms_norm_backward(dy, h, w, 1e-5, dh * mask[:, None], mask)[0]
    assert np.max(np.abs(want - dx)) < 1e-8
