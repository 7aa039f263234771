"""Top alternatives, distillation and embedding: refusals of the C ABI and of the binding, and the oracle's gradients against differences, without a GPU."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2605_07244_amd as m
from paper_2605_07244_amd import binding
from tests import top_oracle as to

P = ctypes.c_void_p
FAKE = P(0x1000)                       # never dereferenced: validation fails first
NO_GPU = (-8, -9)                      # where every argument is right, the call ends at the device check
NAN, INF = float("nan"), float("inf")


def _gpu():
    return torch.cuda.is_available()


def _top(z=FAKE, stride=100, targets=None, mask=None, N=4, V=100, k=5, dt=0, T=1.0, ids=FAKE, top=FAKE, logp=None, lse=None, entropy=None, ws=FAKE, size=1 << 30):
    return m.lib().mrl_top_logprobs(z, stride, targets, mask, N, V, k, dt, T, ids, top, logp, lse, entropy, ws, size, None)


def test_top_argument_errors():
    for bad in (dict(z=None), dict(ids=None, top=None), dict(logp=FAKE), dict(k=0, ids=None, top=None), dict(k=0)):
        assert _top(**bad) == -1, bad
    for bad in (dict(N=-1), dict(N=(1 << 30) + 1), dict(V=0), dict(V=(1 << 24) + 1, stride=1 << 25), dict(stride=99), dict(stride=-1), dict(k=-1), dict(k=101), dict(k=257, V=1000, stride=1000),
                dict(stride=(1 << 40) + 1)):
        assert _top(**bad) == -2, bad
    for dt in (2, -1, 7):
        assert _top(dt=dt) == -3
    for T in (0.0, -1.0, NAN, INF, 1e-5, 2e4):
        assert _top(T=T) == -7
    L = m.lib()
    assert L.mrl_top_logprobs_workspace(4, 100, 5) == 256 and L.mrl_top_logprobs_workspace(4, 100, 257) == 0 and L.mrl_top_logprobs_workspace(-1, 100, 5) == 0
    need = L.mrl_top_logprobs_workspace(4, 100000, 5)
    assert need > 256
    for bad in (dict(ws=None), dict(ws=P(0x1001)), dict(size=need - 1)):
        assert _top(V=100000, stride=100000, **bad) == -6, bad
    assert _top(N=0, z=None, ids=None, top=None, ws=None) == 0
    # what a workgroup per row does needs no workspace
    assert L.mrl_top_logprobs_workspace(2000, 151936, 64) == 256
    if not _gpu():
        assert _top() in NO_GPU and _top(ws=None, N=2000) in NO_GPU and _top(k=0, ids=None, top=None, lse=FAKE) in NO_GPU and _top(ids=None) in NO_GPU


@pytest.mark.parametrize("N,V,k", [(1, 1 << 24, 256), (1, 151936, 1), (3, 151936, 256), (511, 2049, 7), (1023, 50257, 64), (1, 2048, 5), (7, 1 << 24, 0)])
def test_top_workspace_holds_every_part(N, V, k):
    """At most 256 workgroups a row, whose lists together fit into the join's 4096 entries."""
    need = m.lib().mrl_top_logprobs_workspace(N, V, k)
    assert need % 256 == 0 and need <= 512 + N * (256 * 12 + 4096 * 8)


def _distill(h=FAKE, w=FAKE, ids=FAKE, logp=FAKE, mask=None, weight=None, N=4, d=64, V=100, k=5, dt=1, cfg=True, kl=FAKE, dH=FAKE, dW=FAKE, stats=FAKE, ws=FAKE, size=1 << 40, **kw):
    c = m.DistillConfig(**kw).to_c()
    return m.lib().mrl_distill_loss_fwd_bwd(h, w, ids, logp, mask, weight, N, d, V, k, dt, ctypes.byref(c) if cfg else None, kl, dH, dW, stats, ws, size, None)


def test_distill_argument_errors():
    for name in ("h", "w", "ids", "logp", "kl", "stats"):
        assert _distill(**{name: None}) == -1, name
    assert _distill(cfg=False) == -1
    for bad in (dict(N=0), dict(N=-1), dict(N=(1 << 30) + 1), dict(d=0), dict(d=12), dict(V=0), dict(V=(1 << 24) + 1), dict(k=0), dict(k=-1), dict(k=257)):
        assert _distill(**bad) == -2, bad
    for dt in (2, -1):
        assert _distill(dt=dt) == -3
    for bad in (dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=NAN), dict(temperature=INF), dict(temperature=1e-3), dict(temperature=101.0), dict(renormalize=2),
                dict(renormalize=-1), dict(accumulate_dw=2), dict(dh_dtype=2), dict(dw_dtype=2), dict(dw_dtype=1, accumulate_dw=1), dict(dw_dtype=1, dt=0, dh_dtype=0),
                dict(dt=0, dh_dtype=1), dict(chunk_rows=100), dict(chunk_rows=-256), dict(chunk_rows=1 << 21)):
        assert _distill(**bad) == -7, bad
    c = m.DistillConfig()
    for dt in (0, 1):
        assert m.distill_loss_workspace(100, 64, 1000, 5, dt, c) > 0
    assert m.distill_loss_workspace(0, 64, 1000, 5, 1, c) == 0 and m.distill_loss_workspace(100, 64, 1000, 257, 1, c) == 0
    assert m.distill_loss_workspace(100, 64, 1000, 5, 1, m.DistillConfig(temperature=0.0)) == 0
    for bad in (dict(ws=None), dict(ws=P(0x1001)), dict(size=1000)):
        assert _distill(**bad) == -6, bad
    if not _gpu():
        assert _distill() in NO_GPU and _distill(dH=None, dW=None) in NO_GPU and _distill(dt=0, dh_dtype=0, d=7) in NO_GPU and _distill(dw_dtype=1) in NO_GPU


def _look(t=FAKE, ids=FAKE, mask=None, N=4, d=64, V=100, scale=1.0, tt=1, yt=1, y=FAKE):
    return m.lib().mrl_embedding(t, ids, mask, N, d, V, scale, tt, yt, y, None)


def _back(dy=FAKE, ids=FAKE, mask=None, N=4, d=64, V=100, scale=1.0, yt=1, ot=0, acc=0, out=FAKE, ws=FAKE, size=1 << 40):
    return m.lib().mrl_embedding_backward(dy, ids, mask, N, d, V, scale, yt, ot, acc, out, ws, size, None)


def test_embedding_argument_errors():
    for bad in (dict(t=None), dict(ids=None), dict(y=None)):
        assert _look(**bad) == -1, bad
    for bad in (dict(dy=None), dict(ids=None), dict(out=None)):
        assert _back(**bad) == -1, bad
    for bad in (dict(N=-1), dict(N=(1 << 30) + 1), dict(d=0), dict(d=(1 << 20) + 1), dict(V=0), dict(V=(1 << 24) + 1)):
        assert _look(**bad) == -2 and _back(**bad) == -2, bad
    assert _back(N=(1 << 24) + 1) == -2
    for bad in (dict(yt=2), dict(yt=-1)):
        assert _look(**bad) == -3 and _back(**bad) == -3, bad
    assert _look(tt=2) == -3 and _back(ot=2) == -3
    for scale in (NAN, INF, -INF):
        assert _look(scale=scale) == -7 and _back(scale=scale) == -7
    assert _back(acc=2) == -7 and _back(acc=-1) == -7 and _back(acc=1, ot=1) == -7
    need = m.lib().mrl_embedding_backward_workspace(4, 64, 100)
    for bad in (dict(ws=None), dict(ws=P(0x1001)), dict(size=need - 1)):
        assert _back(**bad) == -6, bad
    assert m.lib().mrl_embedding_backward_workspace(1 << 25, 64, 100) == 0
    assert _look(N=0, t=None, ids=None, y=None) == 0 and _back(N=0, dy=None, ids=None, acc=1, ws=None) == 0
    if not _gpu():
        assert _look() in NO_GPU and _back() in NO_GPU and _back(N=0, dy=None, ids=None) in NO_GPU


def test_binding_refusals():
    cpu = torch.zeros(4, 16)
    ids = torch.zeros(4, dtype=torch.int32)
    for f in (lambda: m.top_logprobs(cpu, 3), lambda: m.embedding(cpu, ids), lambda: m.embedding_backward(cpu, ids, 10),
              lambda: m.distill_loss_fwd_bwd(cpu, cpu, torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 3), m.DistillConfig())):
        with pytest.raises(TypeError, match="GPU"):
            f()
    for f in (lambda: m.top_logprobs(cpu[0], 3), lambda: m.top_logprobs(cpu, 1 << 40), lambda: m.embedding(cpu[0], ids), lambda: m.embedding(cpu, ids.view(2, 2)),
              lambda: m.embedding(cpu, ids, out=torch.zeros(3, 16)), lambda: m.embedding_backward(cpu, ids, 1 << 40), lambda: m.embedding_backward(cpu, ids, 10, accumulate=True),
              lambda: m.embedding_backward(cpu, ids, 10, out=torch.zeros(9, 16)),
              lambda: m.distill_loss_fwd_bwd(cpu, torch.zeros(9, 8), torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 3), m.DistillConfig()),
              lambda: m.distill_loss_fwd_bwd(cpu, cpu, torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 2), m.DistillConfig()),
              lambda: m.distill_loss_fwd_bwd(cpu, cpu, torch.zeros(3, 3, dtype=torch.int32), torch.zeros(3, 3), m.DistillConfig()),
              lambda: m.distill_loss_fwd_bwd(cpu, cpu, torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 3), m.DistillConfig(), token_mask=torch.zeros(3, dtype=torch.uint8)),
              lambda: m.distill_loss_fwd_bwd(cpu, cpu, torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 3), m.DistillConfig(accumulate_dw=1))):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: m.embedding(cpu, ids, out_dtype=torch.float16), lambda: m.embedding_backward(cpu, ids, 10, out_dtype=torch.int32),
              lambda: m.embedding(cpu, ids, out=torch.zeros(4, 16), out_dtype=torch.bfloat16), lambda: m.top_logprobs(cpu.half(), 3),
              lambda: m.distill_loss_fwd_bwd(cpu, cpu, torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 3), m.DistillConfig(dw_dtype=2))):
        with pytest.raises(TypeError):
            f()


def test_stats_and_config_have_the_headers_sizes():
    assert ctypes.sizeof(binding._DistillConfig) == 24 and m.binding.DISTILL_STATS_BYTES == 40
    raw = torch.frombuffer(bytearray(np.array([2.5]).tobytes() + np.array([1, 2, 3, 4], dtype=np.int64).tobytes()), dtype=torch.uint8)
    assert m.read_distill_stats(raw) == dict(loss_total=2.5, n_scored_rows=1, n_empty_rows=2, n_saturated_rows=3, n_bad_ids=4)


@pytest.mark.parametrize("renormalize", [False, True])
def test_oracle_gradients_against_differences(renormalize):
    rng = np.random.default_rng(1)
    N, d, V, k, T = 5, 4, 9, 3, 1.7
    h, w, lp = rng.normal(size=(N, d)), rng.normal(size=(V, d)), rng.normal(size=(N, k)) - 2
    ids = rng.integers(-1, V + 1, size=(N, k))
    ids[0] = 4
    mask = np.array([1, 1, 0, 1, 1])
    weight = rng.normal(size=N)
    f = lambda a, b: to.distill(a, b, ids, lp, weight, mask, T, renormalize)[1]
    _, _, dH, dW = to.distill(h, w, ids, lp, weight, mask, T, renormalize)
    e = 1e-6
    for x, g, which in ((h, dH, 0), (w, dW, 1)):
        for at in np.ndindex(*x.shape):
            y = x.copy(), x.copy()
            y[0][at] += e
            y[1][at] -= e
            diff = (f(y[0], w) - f(y[1], w) if which == 0 else f(h, y[0]) - f(h, y[1])) / (2 * e)
            assert abs(diff - g[at]) <= 1e-7 * (1 + abs(g[at]))
    # the library's own: torch on the same
    on = torch.tensor(mask.astype(bool) & ((ids >= 0) & (ids < V)).any(1))
    th, tw = torch.tensor(h, requires_grad=True), torch.tensor(w, requires_grad=True)
    there = torch.tensor((ids >= 0) & (ids < V))
    t = torch.where(there, torch.tensor(lp), torch.tensor(-np.inf, dtype=torch.float64))
    q = torch.softmax(t[on], 1) if renormalize else t[on].exp()
    logq = torch.log(torch.where(q > 0, q, torch.ones_like(q)))
    logp = torch.log_softmax(th @ tw.t() / T, 1)[on].gather(1, torch.tensor(np.clip(ids, 0, V - 1))[on])
    loss = T * T * ((q * (logq - logp)).sum(1) * torch.tensor(weight)[on]).sum()
    loss.backward()
    assert np.allclose(dH, th.grad.numpy(), atol=1e-12) and np.allclose(dW, tw.grad.numpy(), atol=1e-12) and abs(float(loss) - f(h, w)) < 1e-10


def test_oracle_top_against_the_librarys():
    z = torch.randn(6, 50, dtype=torch.float64, generator=torch.Generator().manual_seed(1))
    ids, top, lse, entropy, _ = to.top(z.numpy(), 9, 0.6)
    want = z.topk(9, dim=1)
    assert np.array_equal(ids, want.indices.numpy()) and np.allclose(lse, torch.logsumexp(z / 0.6, 1).numpy())
    assert np.allclose(top, torch.log_softmax(z / 0.6, 1).gather(1, want.indices).numpy())
    assert np.allclose(entropy, torch.distributions.Categorical(logits=z / 0.6).entropy().numpy())
    ties = np.array([[1.0, 2.0, 2.0, -0.0, 0.0, np.nan, -np.inf]])
    assert to.top(ties, 7)[0].tolist() == [[5, 1, 2, 0, 3, 4, 6]]
