"""Top alternatives, distillation loss and embedding in 64 bits, from their definitions."""
import numpy as np
import torch


def f64(t):
    return t.detach().double().cpu().numpy()


def top(z, k, T=1.0):
    """(ids, log-probs of them, lse, entropy, all log-probs) of float64 logits [N, V]; the ids by value, equal ones by the lower, NaN before everything."""
    z = np.asarray(z, dtype=np.float64)
    order = np.empty((z.shape[0], k), dtype=np.int64)
    for n, row in enumerate(z):
        nan = np.isnan(row)
        order[n] = np.lexsort((np.arange(row.size), -np.where(nan, 0.0, row), ~nan))[:k]
    with np.errstate(all="ignore"):
        s = z / T
        m = s.max(1, keepdims=True)
        lse = m + np.log(np.exp(s - m).sum(1, keepdims=True))
        lse = np.where(np.isfinite(m), lse, np.nan)
        logp = s - lse
        p = np.exp(logp)
        entropy = -np.where(p > 0, p * np.where(p > 0, logp, 0.0), 0.0 * lse).sum(1)
    return order, np.take_along_axis(logp, order, 1), lse[:, 0], entropy, logp


def distill(h, w, ids, logp, weight=None, mask=None, T=1.0, renormalize=True):
    """(kl [N], loss, dH, dW) of float64 arrays; ids outside [0, V) are none, rows without any (or without mass, or masked) are left out.  weight None: 1 over the
    number of rows that count."""
    N, V = h.shape[0], w.shape[0]
    there = (ids >= 0) & (ids < V)
    q = np.where(there, np.exp(np.where(there, logp, 0.0) - (np.where(there, logp, -np.inf).max(1, keepdims=True) if renormalize else 0.0)), 0.0)
    with np.errstate(all="ignore"):
        q = np.nan_to_num(q / q.sum(1, keepdims=True)) if renormalize else q
    on = q.sum(1) > 0
    if mask is not None:
        on &= mask != 0
    s = h @ w.T / T
    log_p = s - s.max(1, keepdims=True)
    log_p -= np.log(np.exp(log_p).sum(1, keepdims=True))
    kl, dz = np.zeros(N), np.zeros_like(s)
    c = np.full(N, 1.0 / max(1, on.sum())) if weight is None else weight
    for n in np.nonzero(on)[0]:
        for j in np.nonzero(q[n] > 0)[0]:
            kl[n] += q[n, j] * (np.log(q[n, j]) - log_p[n, ids[n, j]])
            dz[n, ids[n, j]] -= q[n, j]
        dz[n] += q[n].sum() * np.exp(log_p[n])
        dz[n] *= c[n] * T
    return kl, T * T * float(np.sum(np.where(on, c * kl, 0.0))), dz @ w, dz.T @ h


def embedding_backward(dy, ids, V, scale, mask=None):
    """(gradient, sum of magnitudes, rows added) in float64."""
    on = (ids >= 0) & (ids < V)
    if mask is not None:
        on &= mask != 0
    out, mag, count = np.zeros((V, dy.shape[1])), np.zeros((V, dy.shape[1])), np.zeros(V)
    np.add.at(out, ids[on], scale * dy[on])
    np.add.at(mag, ids[on], np.abs(scale * dy[on]))
    np.add.at(count, ids[on], 1)
    return out, mag, count


def rand(shape, dtype, seed, scale=1.0):
    g = torch.Generator("cuda").manual_seed(seed)
    return (scale * torch.randn(shape, device="cuda", generator=g)).to(dtype)
