"""Gradient norm and AdamW against 64 bits: sizes around lanes, blocks and chunks, many tensors, both kinds of moments, and a whole training step of
head and norm.

Bounds.  U = 2^-24.  m is two products and a sum of numbers known to U: 4 U of its terms; v has one more product.  The update's
quotient adds the root (half of v's error, one rounding), a product, the addition of eps and the division: 10 U of itself; p itself is rounded once."""
import numpy as np
import pytest
import torch

from tests import update_oracle as uo
from tests.update_oracle import f64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def mrl():
    import paper_2605_07244_amd as m
    m.lib()
    return m


def _rand(n, seed, scale=1.0, dtype=F32):
    g = torch.Generator("cuda").manual_seed(seed)
    return (scale * torch.randn(n, device="cuda", generator=g)).to(dtype)


def _moments(n, seed, states):
    """Moments of a run under way: (m, v, m_scale, v_scale)."""
    m, root = _rand(n, seed, 3e-4), _rand(n, seed + 1, 1e-3).abs() + 1e-5
    if states == F32:
        return m, root.square(), None, None
    out = []
    for x in (m, root):
        scale = torch.tensor(uo.block_max(f64(x)) / 448 if n else np.zeros(0), dtype=F32, device="cuda")
        out.append(((x / scale.repeat_interleave(256)[:n]).clamp(-448, 448).to(E4M3), scale))
    return out[0][0], out[1][0], out[0][1], out[1][1]


class Set:
    """Tensors of the given sizes, with copies of them as they were."""

    def __init__(self, mrl, sizes, grad=F32, states=F32, copy=True, seed=0, decay=0.01, gap=0):
        self.mrl, self.sizes, self.states = mrl, sizes, states
        at = np.cumsum([0] + [n + gap for n in sizes])

        def parts(flat):
            return [flat[a:a + n] for a, n in zip(at, sizes)]
        total = int(at[-1])
        self.p = parts(_rand(total, seed + 1, 0.02))
        self.g = parts(_rand(total, seed + 2, 1e-3, grad))
        self.copies = parts(torch.zeros(total, dtype=BF16, device="cuda")) if copy else None
        mom = [_moments(n, seed + 10 + 2 * i, states) for i, n in enumerate(sizes)]
        self.m, self.v, ms, vs = (list(x) for x in zip(*mom))
        self.ms, self.vs = (ms, vs) if states == E4M3 else (None, None)
        self.decay = decay if isinstance(decay, list) else [decay] * len(sizes)
        self.plan = mrl.adamw_plan(self.p, self.g, self.copies, self.m, self.v, self.ms, self.vs, weight_decay=decay)
        self.keep()

    def all(self):
        return [*self.p, *self.m, *self.v, *(self.copies or []), *(self.ms or []), *(self.vs or [])]

    def keep(self):
        torch.cuda.synchronize()
        self.old = dict(p=[f64(x) for x in self.p], g=[f64(x) for x in self.g])
        if self.states == F32:
            self.old.update(m=[f64(x) for x in self.m], v=[f64(x) for x in self.v])
        else:
            self.old.update(m=[uo.decode(q, s) for q, s in zip(self.m, self.ms)], v=[uo.decode(q, s) ** 2 for q, s in zip(self.v, self.vs)])

    def check(self, lr, t, coef=1.0, seed=0, b1=0.9, b2=0.999, eps=1e-8):
        torch.cuda.synchronize()
        for i, n in enumerate(self.sizes):
            if n == 0:
                continue
            p0, g, m0, v0 = (self.old[k][i] for k in "pgmv")
            g = g * coef
            p, m, v = uo.adamw(p0, g, m0, v0, lr, t, b1, b2, eps, self.decay[i])
            m_size, v_size = np.abs(b1 * m0) + np.abs((1 - b1) * g), v
            # (decoded 8-bit moments: a product with the scale, and the square of one)
            m_bound, v_bound = 5 * U * m_size, 7 * U * v_size
            root = np.sqrt(v / (1 - b2 ** t)) + eps
            step = lr * (m_size / (1 - b1 ** t) / root * 16 * U + self.decay[i] * np.abs(p0) * 3 * U)
            err = np.abs(f64(self.p[i]) - p)
            assert np.all(err <= U * np.abs(p) + step + 1e-45), (i, n, float(np.max(err / (U * np.abs(p) + step + 1e-45))))
            if self.copies is not None:
                assert torch.equal(self.copies[i], self.p[i].to(BF16)), i
            if self.states == F32:
                assert np.all(np.abs(f64(self.m[i]) - m) <= m_bound + 1e-45), i
                assert np.all(np.abs(f64(self.v[i]) - v) <= v_bound + 1e-45), i
            else:
                bits = uo.random_bits(n, seed, t, i)
                uo.check_codes(f"m of tensor {i}", self.m[i], self.ms[i], m, bits & 0xFFFF, False, rel=4e-6)
                uo.check_codes(f"sqrt(v) of tensor {i}", self.v[i], self.vs[i], np.sqrt(v), bits >> 16, True)


SIZES = [1, 2, 3, 4, 5, 63, 64, 65, 255, 256, 257, 1023, 1024, 1025, 2047, 2048, 2049, 4097, 10001]


@pytest.mark.parametrize("states", [F32, E4M3])
@pytest.mark.parametrize("grad", [F32, BF16])
def test_sizes(mrl, states, grad):
    s = Set(mrl, SIZES, grad, states)
    mrl.adamw_step(s.plan, 1e-3, 5, seed=11)
    s.check(1e-3, 5, seed=11)
    for t in (6, 7):                                     # from what the step before left
        s.keep()
        mrl.adamw_step(s.plan, 3e-4, t, seed=12)
        s.check(3e-4, t, seed=12)


@pytest.mark.parametrize("states", [F32, E4M3])
def test_slices_of_flat_buffers(mrl, states):
    """Tensors one right behind the other at odd offsets, and what lies between them."""
    for gap in (0, 1, 3):
        s = Set(mrl, [5, 1, 259, 2050, 7, 4096, 300], F32, states, gap=gap)
        flat = s.p[0].as_strided((sum(s.sizes) + gap * len(s.sizes),), (1,))
        before = flat.clone()
        mrl.adamw_step(s.plan, 1e-3, 2, seed=3)
        s.check(1e-3, 2, seed=3)
        after, at = flat.clone(), 0
        for n in s.sizes:
            assert torch.equal(before[at + n:at + n + gap], after[at + n:at + n + gap])
            at += n + gap


def test_8_bit_tails_stay_inside_their_tensors(mrl):
    """Codes and scales in guarded buffers: not a byte beside them is written."""
    for n in (1, 2, 3, 5, 255, 257, 2047, 2051):
        m, v, ms, vs = _moments(n, 5, E4M3)
        guards = [torch.full((x.numel() + 64,), 77, dtype=torch.uint8, device="cuda") for x in (m, v)]
        scales = [torch.full((x.numel() + 2,), 7.0, device="cuda") for x in (ms, vs)]
        for g, x in zip(guards, (m, v)):
            g[3:3 + n] = x.view(torch.uint8)
        for g, x in zip(scales, (ms, vs)):
            g[1:-1] = x
        p, g = _rand(n, 1), _rand(n, 2, 1e-3)
        copy = torch.full((n + 4,), 5.0, dtype=BF16, device="cuda")
        codes = [x[3:3 + n].view(E4M3) for x in guards]
        plan = mrl.adamw_plan([p], [g], [copy[1:1 + n]], [codes[0]], [codes[1]], [scales[0][1:-1]], [scales[1][1:-1]])
        mrl.adamw_step(plan, 1e-3, 9, seed=4)
        p2 = _rand(n, 1)
        plan2 = mrl.adamw_plan([p2], [g], None, [m], [v], [ms], [vs])
        mrl.adamw_step(plan2, 1e-3, 9, seed=4)
        torch.cuda.synchronize()
        assert torch.equal(p, p2) and torch.equal(copy[1:1 + n], p.to(BF16)) and copy[0] == 5 and bool((copy[1 + n:] == 5).all())
        for g, x in zip(guards, (m, v)):
            assert torch.equal(g[3:3 + n], x.view(torch.uint8)) and bool((g[:3] == 77).all()) and bool((g[3 + n:] == 77).all())
        for g, x in zip(scales, (ms, vs)):
            assert torch.equal(g[1:-1], x) and g[0] == 7 and g[-1] == 7


@pytest.mark.parametrize("states", [F32, E4M3])
def test_many_tensors(mrl, states):
    """More tensors than a launch takes, empty ones among them, a weight decay for each; as many calls of one tensor give the same."""
    sizes = [(37 * i) % 1500 for i in range(203)]
    decay = [0.01 * (i % 3) for i in range(203)]
    s = Set(mrl, sizes, F32, states, decay=decay)
    assert sizes.count(0) >= 1
    mrl.adamw_step(s.plan, 1e-3, 4, seed=5)
    s.check(1e-3, 4, seed=5)
    coef = mrl.grad_norm(s.plan, 0.01)
    norm, c = uo.grad_norm([f64(x) for x in s.g], 0.01)
    assert abs(float(coef[0]) - norm) <= 2 * U * norm and abs(float(coef[1]) - c) <= 2 * U * c


@pytest.mark.parametrize("sizes,grad", [([1], F32), ([2049], BF16), ([3, 70001, 0, 5], F32), ([2048 * 1024 + 1], F32), ([5000000, 33], BF16), ([100] * 300, F32), ([0], F32)])
def test_grad_norm(mrl, sizes, grad):
    g = [_rand(n, i, 1e-3 * (1 + i % 5), grad) for i, n in enumerate(sizes)]
    plan = mrl.grad_plan(g)
    norm, _ = uo.grad_norm([f64(x) for x in g], 1.0)
    for most in (float("inf"), 1.0, 0.5 * norm, norm * 2) if norm else (1.0,):
        got = mrl.grad_norm(plan, most)
        # exact squares, sums in fp64, one rounding to fp32
        assert abs(float(got[0]) - norm) <= 1.001 * U * norm
        want = min(1.0, most / norm) if norm else 1.0
        assert abs(float(got[1]) - want) <= 1.001 * U * want
        assert torch.equal(got, mrl.grad_norm(plan, most))


def test_grad_norm_of_large_small_and_no_numbers(mrl):
    """Squares that overflow and underflow fp32 are sums in fp64; what is no number is said so, wherever it lies."""
    big, small = torch.full((5000,), 3e38, device="cuda"), torch.full((5000,), 1e-30, device="cuda")
    got = mrl.grad_norm(mrl.grad_plan([big]), 1.0)
    # the norm, 2.1e40, is above fp32; its inverse 4.714e-41 is a subnormal, known to half of 2^-149: 7.0e-46 / 4.714e-41 = 1.49e-5 of itself
    assert float(got[0]) == float("inf") and abs(float(got[1]) * 3e38 * 5000 ** 0.5 - 1) < 1.5e-5
    got = mrl.grad_norm(mrl.grad_plan([small]), 1.0)
    assert abs(float(got[0]) / (1e-30 * 5000 ** 0.5) - 1) < 1e-6 and float(got[1]) == 1.0
    for odd in (float("nan"), float("inf"), -float("inf")):
        for at in (0, 2048, 4999):
            g = _rand(5000, 1)
            g[at] = odd
            got = mrl.grad_norm(mrl.grad_plan([_rand(77, 2), g]), 1.0)
            assert not np.isfinite(float(got[0])) and np.isnan(float(got[1]))
    none = mrl.grad_norm(mrl.grad_plan([]), 1.0)
    assert none.tolist() == [0.0, 1.0]


@pytest.mark.parametrize("states", [F32, E4M3])
def test_clipped_and_skipped(mrl, states):
    s = Set(mrl, [700, 3000], F32, states)
    norm, c = uo.grad_norm(s.old["g"], 0.01)
    coef = mrl.grad_norm(s.plan, 0.01)
    mrl.adamw_step(s.plan, 1e-3, 3, norm_coef=coef, seed=1, skip_nonfinite=True)
    s.check(1e-3, 3, coef=c, seed=1)
    s.g[1][2999] = float("nan")
    before = [x.clone() for x in s.all()]
    coef = mrl.grad_norm(s.plan, 0.01)
    mrl.adamw_step(s.plan, 1e-3, 4, norm_coef=coef, seed=1, skip_nonfinite=True)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, s.all()))
    # without a coefficient, a NaN spoils its element or its block of 8-bit moments, and nothing else
    mrl.adamw_step(s.plan, 1e-3, 4, seed=1)
    assert bool(s.p[1][2999].isnan()) and int(s.p[1].isnan().sum()) == 1 and not bool(s.p[0].isnan().any())
    m = s.m[1] if states == F32 else torch.tensor(uo.decode(s.m[1], s.ms[1]))
    v = s.v[1] if states == F32 else torch.tensor(uo.decode(s.v[1], s.vs[1]))
    lost = 1 if states == F32 else 3000 - 11 * 256
    assert int(m.isnan().sum()) == lost and int(v.isnan().sum()) == lost


@pytest.mark.parametrize("states", [F32, E4M3])
def test_from_nothing(mrl, states):
    """The first step of a new run: moments that the plan allocates, zero gradients among the others."""
    p, g = _rand(3000, 1, 0.02), _rand(3000, 2, 1e-3)
    g[:700] = 0.0
    p0, copy = p.clone(), torch.empty(3000, dtype=BF16, device="cuda")
    plan = mrl.adamw_plan([p], [g], [copy], state_dtype=states, weight_decay=0.0)
    mrl.adamw_step(plan, 1e-3, 1)
    torch.cuda.synchronize()
    assert torch.equal(p[:700], p0[:700]) and torch.equal(copy, p.to(BF16))
    # m / (1 - b1) = g and v / (1 - b2) = g^2: a step of lr each
    want = f64(p0) - 1e-3 * f64(g) / (np.abs(f64(g)) + 1e-8)
    assert np.all(np.abs(f64(p) - want) <= U * np.abs(want) + 1e-3 * 20 * U)
    if states == E4M3:
        assert float(uo.decode(plan.v[0], plan.v_scale[0])[700:].min()) > 0 and not uo.decode(plan.v[0], plan.v_scale[0])[:700].any()


def test_8_bit_moments_follow_those_of_32_bits(mrl):
    """After 3000 steps of gradients of steady size: sqrt(v) is right on average (rounded to nearest, its codes would have stopped after a few
    steps, an error of 0.9 and more), and single values scatter by no more than a code's step."""
    n = 256 * 64
    sigma = 1e-3 * torch.exp(1.5 * _rand(n, 1))
    g = torch.empty(n, device="cuda")
    gen = torch.Generator("cuda").manual_seed(3)
    plans = [mrl.adamw_plan([torch.zeros(n, device="cuda")], [g], state_dtype=t, weight_decay=0.0) for t in (F32, E4M3)]
    for t in range(1, 3001):
        torch.randn(n, device="cuda", generator=gen, out=g)
        g.mul_(sigma)
        for plan in plans:
            mrl.adamw_step(plan, 1e-3, t, seed=9)
    root = f64(plans[0].v[0]) ** 0.5
    got = uo.decode(plans[1].v[0], plans[1].v_scale[0])
    large = root > 1e-3 * np.repeat(uo.block_max(root), 256)          # (well inside the normal codes)
    ratio = got[large] / root[large]
    # codes are at most 1/8 apart; of single steps' roundings, b2^i of each remains: 1/8 / sqrt(12 (1 - b2^2)) would be 0.8 for
    # independent roundings that nothing restores, but a wrong root is pulled back by the same 0.1 % a step that moves it
    print("sqrt(v), 8 bits over 32: mean", ratio.mean(), "deviation", ratio.std())
    assert abs(ratio.mean() - 1) < 0.1


def test_numbers_from_the_device_and_replays(mrl):
    """A captured step takes its learning rate and step from the device; eager calls of the same steps give the same bits."""
    for states in (F32, E4M3):
        a, b = Set(mrl, [1000, 5000], F32, states), Set(mrl, [1000, 5000], F32, states)
        lr, step = torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            mrl.grad_norm(a.plan, 0.01)                  # (the first call of a process loads the kernels)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step.add_(1)
            coef = mrl.grad_norm(a.plan, 0.01)
            mrl.adamw_step(a.plan, lr, step, norm_coef=coef, seed=21, skip_nonfinite=True)
        for t in range(1, 5):
            lr.fill_(1e-3 / t)
            for k in range(2):
                a.g[k].copy_(_rand(a.sizes[k], 50 * t + k, 1e-3))
                b.g[k].copy_(a.g[k])
            if t == 3:
                a.g[0][5] = b.g[0][5] = float("inf")     # skipped
            graph.replay()
            torch.cuda.synchronize()
            mrl.adamw_step(b.plan, float(lr), t, norm_coef=mrl.grad_norm(b.plan, 0.01), seed=21, skip_nonfinite=True)
            assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a.all(), b.all())), t


def test_more_than_2_33_elements(mrl):
    """One tensor whose offsets pass 32 bits, and whose workgroups pass what a launch takes along x: its end is updated as a tensor of its own would be, with
    the random bits of its places."""
    n, k = 2 ** 33 + 3 * 2048 + 301, 5000
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=BF16, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2))
    ms, vs = (torch.zeros(-(-n // 256), device="cuda") for _ in range(2))
    g[-k:] = _rand(k, 1, 1e-3, BF16)
    plan = mrl.adamw_plan([p], [g], None, [m], [v], [ms], [vs])
    got = mrl.grad_norm(plan, 1e-3)
    norm, c = uo.grad_norm([f64(g[-k:])], 1e-3)
    assert abs(float(got[0]) - norm) <= 1.001 * U * norm
    mrl.adamw_step(plan, 1e-3, 1, seed=6)
    torch.cuda.synchronize()
    first = (n - k) // 256 * 256                         # a block's beginning
    grad = f64(g[first:])
    want, m1, v1 = uo.adamw(np.zeros(n - first), grad, np.zeros(n - first), np.zeros(n - first), 1e-3, 1)
    assert np.all(np.abs(f64(p[first:]) - want) <= 21 * U * 1e-3)
    bits = uo.random_bits(n - first, 6, 1, 0, first)
    uo.check_codes("m", m[first:], ms[first // 256:], m1, bits & 0xFFFF, False)
    uo.check_codes("sqrt(v)", v[first:], vs[first // 256:], np.sqrt(v1), bits >> 16, True)
    assert not bool(p[:2 ** 20].any()) and not bool(p[2 ** 31 - 1000:2 ** 31 + 1000].any())


def test_threads_on_streams_of_their_own(mrl):
    """Calls of several host threads at once, each on its own stream and data, give what the same calls give one after the other."""
    import threading

    def work(k, out):
        g = torch.Generator("cuda").manual_seed(k)
        N, d = 700 + 300 * k, 513 + 64 * k
        x, w = torch.randn((N, d), device="cuda", generator=g), 1 + 0.1 * torch.randn(d, device="cuda", generator=g)
        p, grad = [w.clone(), x.reshape(-1).clone()], [torch.empty(d, device="cuda"), torch.empty(N * d, device="cuda")]
        plan = mrl.adamw_plan(p, grad, state_dtype=E4M3 if k % 2 else F32)
        for t in range(1, 6):
            y, h, _ = mrl.rms_norm(p[1].view(N, d), p[0], 1e-5, x)
            dx, _ = mrl.rms_norm_backward(y, h, p[0], 1e-5, out_dweight=grad[0])
            grad[1].copy_(dx.reshape(-1))
            mrl.adamw_step(plan, 1e-3, t, norm_coef=mrl.grad_norm(plan, 1.0), seed=k)
        torch.cuda.current_stream().synchronize()
        out[k] = [x.clone() for x in (*p, *plan.m, *plan.v)]

    alone, together = {}, {}
    for k in range(4):
        work(k, alone)

    def on_a_stream(k):
        with torch.cuda.stream(torch.cuda.Stream()):
            work(k, together)
    torch.cuda.synchronize()
    threads = [threading.Thread(target=on_a_stream, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for k in range(4):
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(alone[k], together[k])), k


def test_refusals(mrl):
    p, g = torch.zeros(10, device="cuda"), torch.zeros(10, device="cuda")
    for bad in (lambda: mrl.adamw_plan([p.bfloat16()], [g]), lambda: mrl.adamw_plan([p], [g.half()]), lambda: mrl.adamw_plan([p], [g], [p]),
                lambda: mrl.adamw_plan([p], [g], state_dtype=BF16), lambda: mrl.adamw_plan([p], [g], m=[p.bfloat16()], state_dtype=F32),
                lambda: mrl.grad_plan([p.double()])):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: mrl.adamw_plan([p], [g[:9]]), lambda: mrl.adamw_plan([p, p], [g]), lambda: mrl.adamw_plan([p], [g], weight_decay=[0.1, 0.1]),
                lambda: mrl.adamw_plan([p], [g], m=[]), lambda: mrl.grad_plan([torch.zeros(8, 8, device="cuda").t()]),
                lambda: mrl.adamw_plan([p], [g], state_dtype=E4M3, m_scale=[torch.zeros(2, device="cuda")]),
                lambda: mrl.adamw_plan([p], [g], m=[torch.zeros(10, device="cuda").to(E4M3)]),
                lambda: mrl.adamw_plan([p], [g], m=[torch.zeros(10, device="cuda").to(E4M3)], m_scale=[torch.zeros(2, device="cuda")])):
        with pytest.raises(ValueError):
            bad()
    plan = mrl.adamw_plan([p], [g])
    for bad in (lambda: mrl.adamw_plan([p, p], [g, g]), lambda: mrl.adamw_plan([p], [p]), lambda: mrl.adamw_plan([p], [g], weight_decay=-1.0),
                lambda: mrl.adamw_step(plan, -1.0, 1), lambda: mrl.adamw_step(plan, 1e-3, 0), lambda: mrl.adamw_step(plan, 1e-3, 1, beta1=1.0),
                lambda: mrl.grad_norm(plan, 0.0)):
        with pytest.raises(mrl.MrlError) as e:
            bad()
        assert e.value.status == -7
    for bad in (lambda: mrl.adamw_step(plan, torch.zeros(2, device="cuda"), 1), lambda: mrl.adamw_step(plan, 1e-3, 1, norm_coef=torch.zeros(1, device="cuda")),
                lambda: mrl.grad_norm(plan, 1.0, out=torch.zeros(3, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        mrl.adamw_step(plan, torch.zeros(1, device="cuda", dtype=torch.float64), 1)


def test_a_training_step_of_head_and_norm(mrl):
    """Norm, scoring loss, both backward passes, clipping and update, as they follow one another, against the same chain in 64 bits."""
    from oracle import mrl_oracle as orc
    from tests import util
    from workloads import synth
    sp = synth.spec(2, n_prompts=2, T=24, V=1200)
    b = synth.make(sp, "cuda")
    N, d = b["H"].shape
    V = b["W"].shape[0]
    mask = b["mask"].reshape(-1)
    x, res = b["H"], _rand(N * d, 3, 0.5, BF16).view(N, d)
    norm_w, head = 1 + _rand(d, 4, 0.1), b["W"].float()
    norm16, head16 = norm_w.to(BF16), b["W"].clone()
    dhead, dnorm = torch.empty(V, d, device="cuda"), torch.empty(d, device="cuda")
    adv, *_ = mrl.group_advantages(b["rewards_all"], b["group_all"], b["G"], b["in_stats"], b["scored"], b["is_own"])
    seq_adv = synth.seq_adv_from(adv, b)
    lc = mrl.LossConfig(kl_beta=sp.kl_beta, sgt_lambda=sp.sgt_lambda)
    cfg = util.cfg_dict(sp)
    # the oracle's chain, from the bf16 hidden states and gradients that the path hands on
    m = mask.cpu().numpy()
    y0, h0 = uo.rms_norm(f64(x), f64(norm16), EPS := 1e-5, f64(res), m)
    H, h, _ = mrl.rms_norm(x, norm16, EPS, residual=res, token_mask=mask)
    assert np.all(np.abs(f64(H) - y0) <= (2.0 ** -8 + 52 * U) * np.abs(y0))
    b["H"] = H
    first = util.oracle_loss(b, seq_adv.cpu().numpy(), cfg, need_grads=False)
    b["behav"] = util.move_off_kinks(b, first["logp"], sp.clip_eps)
    want = util.oracle_loss(b, seq_adv.cpu().numpy(), cfg)
    for states in (F32, E4M3):
        p, p16 = [head.clone(), norm_w.clone()], [head16.clone(), norm16.clone()]
        plan = mrl.adamw_plan(p, [dhead, dnorm], p16, state_dtype=states, weight_decay=[0.01, 0.0])
        out = mrl.grpo_loss_fwd_bwd(H, p16[0], b["targets"], mask, b["behav"], b["ref"], seq_adv, b["seq_group"], b["seq_kind"], b["B"], b["T"], b["G"],
                                    lc, out_dW=dhead)
        dx, _ = mrl.rms_norm_backward(out["dH"], h, p16[1], EPS, token_mask=mask, out_dweight=dnorm)
        coef = mrl.grad_norm(plan, 0.1)
        mrl.adamw_step(plan, 1e-3, 1, norm_coef=coef, seed=1, skip_nonfinite=True)
        torch.cuda.synchronize()
        dx_o, dn_o, *_ = uo.rms_norm_backward(want["dH"], f64(h), f64(norm16), EPS, None, m)
        assert util.rel_fro(f64(dx), dx_o) <= util.REL_TOL and util.rel_fro(f64(dnorm), dn_o) <= util.REL_TOL
        assert util.rel_fro(f64(dhead), want["dW"]) <= util.REL_TOL
        norm_o, coef_o = uo.grad_norm([want["dW"], dn_o], 0.1)
        assert abs(float(coef[0]) - norm_o) <= util.REL_TOL * norm_o
        # the update from the path's own gradients: each stage is held to its inputs
        for p_new, p_old, g, decay, c16 in ((p[0], head, dhead, 0.01, p16[0]), (p[1], norm_w, dnorm, 0.0, p16[1])):
            gc = f64(g).reshape(-1) * float(coef[1])
            p_o, m_o, v_o = uo.adamw(f64(p_old).reshape(-1), gc, 0 * gc, 0 * gc, 1e-3, 1, decay=decay)
            assert np.all(np.abs(f64(p_new).reshape(-1) - p_o) <= U * np.abs(p_o) + 1e-3 * 24 * U)
            assert torch.equal(c16, p_new.to(BF16))


@pytest.mark.parametrize("n", [700, 512, 256, 3])
@pytest.mark.parametrize("odd", [float("inf"), -float("inf"), float("nan"), 1e21])
def test_8_bit_moments_of_no_numbers(mrl, n, odd):
    """A gradient that is not finite makes both 8-bit moments of its block NaN, one whose square is not (1e-3 * 1e42 is above 3.4e38) the second: a scale
    that is infinite instead would leave v infinite, and an infinite v holds the block's weights where they are, for good and without a sign of it.  Other blocks do not see it."""
    at = n - 1 if n < 512 else 300
    block = slice(at // 256 * 256, min(at // 256 * 256 + 256, n))
    g = _rand(n, 2, 1e-3)
    sets = []
    for spoiled in (False, True):
        m, v, ms, vs = _moments(n, 5, E4M3)
        grad = g.clone()
        if spoiled:
            grad[at] = odd
        p = _rand(n, 1, 0.02)
        sets.append((p, grad, mrl.adamw_plan([p], [grad], None, [m], [v], [ms], [vs])))
    for t in (5, 6):
        for p, grad, plan in sets:
            mrl.adamw_step(plan, 1e-3, t, seed=3)
        torch.cuda.synchronize()
        (p0, _, clean), (p1, _, plan) = sets
        m, root = uo.decode(plan.m[0], plan.m_scale[0]), uo.decode(plan.v[0], plan.v_scale[0])
        assert np.all(np.isnan(root[block])), (t, int(np.isinf(root).sum()))
        assert np.all(np.isnan(m[block])) if not np.isfinite(odd) else np.all(np.isfinite(m[block]))
        rest = np.ones(n, dtype=bool)
        rest[block] = False
        assert np.array_equal(m[rest], uo.decode(clean.m[0], clean.m_scale[0])[rest]) and np.array_equal(root[rest], uo.decode(clean.v[0], clean.v_scale[0])[rest])
        assert np.array_equal(f64(p1)[rest], f64(p0)[rest])
        if t == 6:
            assert np.all(np.isnan(f64(p1)[block]))


def test_copies_of_some_tensors(mrl):
    """None in a list of copies: that tensor has none, the others' are written, and the weights are those of a plan without any."""
    sizes = [5, 300, 1000]
    for states in (F32, E4M3):
        a, b = Set(mrl, sizes, F32, states, copy=False), Set(mrl, sizes, F32, states, copy=False)
        copies = [None, torch.empty(300, dtype=BF16, device="cuda"), None]
        plan = mrl.adamw_plan(a.p, a.g, copies, a.m, a.v, a.ms, a.vs, weight_decay=0.01)
        mrl.adamw_step(plan, 1e-3, 2, seed=8)
        mrl.adamw_step(b.plan, 1e-3, 2, seed=8)
        torch.cuda.synchronize()
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a.all(), b.all()))
        assert torch.equal(copies[1], a.p[1].to(BF16))
        with pytest.raises(ValueError):
            mrl.adamw_plan(a.p, a.g, copies[:2], a.m, a.v, a.ms, a.vs)
        with pytest.raises(ValueError):
            mrl.adamw_plan(a.p, a.g, [None, copies[1][:299], None], a.m, a.v, a.ms, a.vs)
        for bad in (dict(params=[a.p[0], None, a.p[2]]), dict(v=[a.v[0], None, a.v[2]])):
            with pytest.raises(TypeError, match="must hold tensors"):
                mrl.adamw_plan(**(dict(params=a.p, grads=a.g, m=a.m, v=a.v, m_scale=a.ms, v_scale=a.vs) | bad))


@pytest.mark.parametrize("states", [F32, E4M3])
def test_a_plan_holds_on_to_its_memory(mrl, states):
    """Tensors that were given other memory since, and moments replaced in the plan's lists: what the plan still writes to belongs to nobody else."""
    n = 3 << 20                                          # (large enough for blocks of their own, which the allocator would hand out again)
    s = Set(mrl, [n], F32, states)
    plan = s.plan
    lists = [x for x in (plan.params, plan.grads, plan.copies, plan.m, plan.v, plan.m_scale, plan.v_scale) if x]
    old = [x[0].data_ptr() for x in lists]
    for k, x in enumerate(lists):
        if k % 2:
            x[0].data = x[0].clone()
        x[0] = x[0].clone()
    del s
    torch.cuda.synchronize()
    others = [torch.full((size,), 7, dtype=torch.uint8, device="cuda") for size in (4 * n, 2 * n, n, n // 64) for _ in range(8)]
    assert not {x.data_ptr() for x in others} & set(old)
    mrl.adamw_step(plan, 1e-3, 1, norm_coef=mrl.grad_norm(plan, 1.0), seed=1)
    torch.cuda.synchronize()
    assert all(bool((x == 7).all()) for x in others)


def test_scatter_of_8_bit_moments(mrl):
    """sqrt(v) in codes against 32 bits after 3000 steps of steady gradients: not only the mean is held, so that errors of two halves do not cancel.

    Relative to r = sqrt(v), a step moves it by 5e-4 (z^2 - 1), z normal, and the block's scale moves by as much of another element; codes lie s = 1/16 to 1/8 of r
    apart, 0.090 in the mean over the logarithm.  A value that lies f steps off a code is rounded with a variance of f s^2 at most, f s = 5e-4 |z1^2 - z2^2|, whose
    mean is 5e-4 * 4 / pi = 6.4e-4.  A root that is off by x is pulled back by 1e-3 x a step: the variance settles at 6.4e-4 s / (2 * 1e-3) = 0.32 s, a deviation of 0.17
    (0.20 where s is 1/8).  Held: a deviation below 0.22 and above 0.12, and 99 % of the values within 0.7, 3.5 times the larger of the two.
    The mean moves with the variance alone, by (1.5 times) it at most: 0.05 (pulled back are squares), and by 5 / sqrt(16384) * 0.2 of chance."""
    n = 256 * 64
    sigma = 1e-3 * torch.exp(1.5 * _rand(n, 21))
    g = torch.empty(n, device="cuda")
    gen = torch.Generator("cuda").manual_seed(23)
    plans = [mrl.adamw_plan([torch.zeros(n, device="cuda")], [g], state_dtype=t, weight_decay=0.0) for t in (F32, E4M3)]
    for t in range(1, 3001):
        torch.randn(n, device="cuda", generator=gen, out=g)
        g.mul_(sigma)
        for plan in plans:
            mrl.adamw_step(plan, 1e-3, t, seed=31)
    root = f64(plans[0].v[0]) ** 0.5
    got = uo.decode(plans[1].v[0], plans[1].v_scale[0])
    large = root > 1e-3 * np.repeat(uo.block_max(root), 256)          # (well inside the normal codes)
    off = got[large] / root[large] - 1
    far = np.quantile(np.abs(off), 0.99)
    print(f"{large.sum()} values: mean {off.mean():.4f} deviation {off.std():.4f} 99 % within {far:.3f}")
    assert large.sum() > n // 2
    assert abs(off.mean()) <= 0.06 and 0.12 <= off.std() <= 0.22 and far <= 0.7


@pytest.mark.parametrize("states", [F32, E4M3])
@pytest.mark.parametrize("b1,b2", [(0.9, 0.999), (0.0, 0.0), (0.0, 0.95)])
def test_gradients_of_both_types_in_one_plan(mrl, states, b1, b2):
    """Tensors with float and bfloat16 gradients side by side, more of them than a word of their flags has bits; betas of zero, under which a moment is its gradient."""
    sizes = [1 + (97 * i) % 700 for i in range(70)]
    s = Set(mrl, sizes, F32, states)
    s.g = [g.to(BF16) if i % 3 == 1 else g for i, g in enumerate(s.g)]
    s.plan = mrl.adamw_plan(s.p, s.g, s.copies, s.m, s.v, s.ms, s.vs, weight_decay=0.01)
    s.keep()
    norm, c = uo.grad_norm(s.old["g"], 1e-3)
    got = mrl.grad_norm(s.plan, 1e-3)
    assert abs(float(got[0]) - norm) <= 1.001 * U * norm and abs(float(got[1]) - c) <= 1.001 * U * c
    mrl.adamw_step(s.plan, 1e-3, 3, beta1=b1, beta2=b2, norm_coef=got, seed=6)
    s.check(1e-3, 3, coef=float(got[1]), seed=6, b1=b1, b2=b2)


@pytest.mark.parametrize("states", [F32, E4M3])
def test_a_number_beside_one_from_the_device(mrl, states):
    """Learning rate or step alone from the device, and steps below 1 there, which count as 1: the same bits as with numbers."""
    def after(lr, step):
        s = Set(mrl, [300, 1000], F32, states)
        mrl.adamw_step(s.plan, lr, step, seed=9)
        torch.cuda.synchronize()
        return s.all()
    lr = torch.full((1,), 1e-3, device="cuda")
    rate = float(lr)                                     # (what the tensor holds, to the bit)
    for step in (1, 2, 1000, (1 << 32) + 3):
        want = after(rate, step)
        on_device = torch.full((1,), step, dtype=torch.int64, device="cuda")
        for got in (after(lr, step), after(rate, on_device), after(lr, on_device)):
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(want, got)), step
    want = after(rate, 1)
    for step in (0, -1, -(1 << 40)):
        got = after(lr, torch.full((1,), step, dtype=torch.int64, device="cuda"))
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(want, got)), step
