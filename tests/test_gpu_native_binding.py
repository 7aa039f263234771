"""The calls whose host side is native give through ctypes what they give through it, bit for bit, and their refusals are the same."""
import pytest
import torch

from paper_2605_07244_amd import binding
from tests.top_oracle import rand

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def mrl():
    import paper_2605_07244_amd as m
    m.lib()
    return m


def _calls(mrl):
    g = torch.Generator("cuda").manual_seed(1)
    ints = lambda n, *shape: torch.randint(-1, n, shape, device="cuda", generator=g, dtype=torch.int32)
    mask = (torch.arange(50, device="cuda") % 3 != 0).to(torch.uint8)
    z, wide, y = rand((50, 1000), BF16, 1, 3.0), rand((50, 1013), F32, 2, 3.0), ints(1000, 50)
    table, dy, ids = rand((300, 72), BF16, 3), rand((50, 72), F32, 4), ints(300, 50)
    h, w, ti, tl = rand((50, 72), BF16, 5), rand((300, 72), BF16, 6, 0.3), ints(300, 50, 9), -torch.rand(50, 9, device="cuda", generator=g)
    weight = torch.rand(50, device="cuda", generator=g)
    one = rand((1, 100000), F32, 7, 3.0)
    return [
        lambda: mrl.top_logprobs(z, 7),
        lambda: mrl.top_logprobs(z, 7, y, mask, 2.0),
        lambda: mrl.top_logprobs(wide[:, 5:1005], 30, y, want_lse=False, want_entropy=False),
        lambda: mrl.top_logprobs(z, 0, y),
        lambda: mrl.top_logprobs(one, 64),
        lambda: mrl.embedding(table, ids),
        lambda: mrl.embedding(table, ids, 3.0, mask, F32),
        lambda: mrl.embedding_backward(dy, ids, 300),
        lambda: mrl.embedding_backward(dy, ids, 300, 0.25, mask, BF16),
        lambda: mrl.distill_loss_fwd_bwd(h, w, ti, tl, mrl.DistillConfig()),
        lambda: mrl.distill_loss_fwd_bwd(h, w, ti, tl, mrl.DistillConfig(2.0, 0, 0, mrl.F32, mrl.BF16), token_mask=mask, row_weight=weight),
        lambda: mrl.distill_loss_fwd_bwd(h, w, ti, tl, mrl.DistillConfig(), want_dH=False, want_dW=False),
    ]


def _leaves(r):
    return [r[k] for k in sorted(r)] if isinstance(r, dict) else [r]


def test_both_ways_give_the_same(mrl, monkeypatch):
    assert binding._host() is not binding._NoHost
    for f in _calls(mrl):
        monkeypatch.setattr(binding, "_native", True)
        a = _leaves(f())
        monkeypatch.setattr(binding, "_native", False)
        b = _leaves(f())
        assert len(a) == len(b)
        for x, y in zip(a, b):
            assert (x is None) == (y is None)
            assert x is None or (x.dtype == y.dtype and x.shape == y.shape and torch.equal(x, y))


@pytest.mark.parametrize("native", [True, False])
def test_refusals(mrl, monkeypatch, native):
    monkeypatch.setattr(binding, "_native", native)
    z = rand((4, 100), F32, 1)
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    h, w = rand((4, 64), BF16, 1), rand((100, 64), BF16, 2)
    ti, tl = torch.zeros(4, 3, dtype=torch.int32, device="cuda"), torch.zeros(4, 3, device="cuda")
    cfg = mrl.DistillConfig()
    wrong = [
        (ValueError, lambda: mrl.top_logprobs(z.t(), 3)),
        (ValueError, lambda: mrl.top_logprobs(z[:1].expand(4, 100), 3)),
        (ValueError, lambda: mrl.top_logprobs(z, 3, target_ids=ids[:3])),
        (TypeError, lambda: mrl.top_logprobs(z, 3, target_ids=ids.long())),
        (TypeError, lambda: mrl.top_logprobs(z.half(), 3)),
        (TypeError, lambda: mrl.top_logprobs(z, 2.5)),
        (mrl.MrlError, lambda: mrl.top_logprobs(z, 101)),
        (ValueError, lambda: mrl.top_logprobs(z[0], 3)),
        (mrl.MrlError, lambda: mrl.top_logprobs(z, 3, temperature=0.0)),
        (mrl.MrlError, lambda: mrl.top_logprobs(z, 0, want_lse=False, want_entropy=False)),
        (ValueError, lambda: mrl.embedding(w.t(), ids)),
        (TypeError, lambda: mrl.embedding(w, ids.long())),
        (ValueError, lambda: mrl.embedding(w, ids, token_mask=torch.ones(3, dtype=torch.uint8, device="cuda"))),
        (mrl.MrlError, lambda: mrl.embedding(w, ids, float("nan"))),
        (ValueError, lambda: mrl.embedding_backward(h.t(), ids, 100)),
        (ValueError, lambda: mrl.embedding_backward(h, ids[:3], 100)),
        (mrl.MrlError, lambda: mrl.embedding_backward(h, ids, 0)),
        (mrl.MrlError, lambda: mrl.embedding_backward(h, ids, 100, out=torch.zeros(100, 64, device="cuda", dtype=BF16), accumulate=True)),
        (mrl.MrlError, lambda: mrl.embedding_backward(h, ids, 100, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))),
        (ValueError, lambda: mrl.distill_loss_fwd_bwd(h, w, ti[:3], tl, cfg)),
        (TypeError, lambda: mrl.distill_loss_fwd_bwd(h, w, ti.long(), tl, cfg)),
        (TypeError, lambda: mrl.distill_loss_fwd_bwd(h, w, ti, tl.bfloat16(), cfg)),
        (ValueError, lambda: mrl.distill_loss_fwd_bwd(h, w.float(), ti, tl, cfg)),
        (mrl.MrlError, lambda: mrl.distill_loss_fwd_bwd(h, w, ti, tl, mrl.DistillConfig(temperature=0.0))),
        (mrl.MrlError, lambda: mrl.distill_loss_fwd_bwd(h.float(), w.float(), ti, tl, cfg)),
        (mrl.MrlError, lambda: mrl.distill_loss_fwd_bwd(h[:0], w, ti[:0], tl[:0], cfg)),
        (TypeError, lambda: mrl.distill_loss_fwd_bwd(h, w, ti, tl, cfg, out_dW=torch.zeros(100, 64, device="cuda", dtype=BF16))),
        (ValueError, lambda: mrl.distill_loss_fwd_bwd(h, w, ti, tl, cfg, out_stats=torch.zeros(39, device="cuda", dtype=torch.uint8))),
    ]
    for kind, f in wrong:
        with pytest.raises(kind):
            f()
