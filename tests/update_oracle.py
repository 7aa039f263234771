"""Norm, its backward, gradient norm and AdamW in 64 bits, from their formulas."""
import numpy as np
import torch

E4M3_MAX, LEAST = 448.0, 2.0 ** -100


def f64(t):
    """float64 copy of a float32, bfloat16 or float8_e4m3fn tensor."""
    return t.detach().cpu().float().numpy().astype(np.float64)


def rms_norm(x, w, eps, residual=None, mask=None):
    """(y, h), h and y of rows with mask 0 zero."""
    h = x + residual if residual is not None else x.copy()
    if mask is not None:
        h[mask == 0] = 0.0
    return h / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps) * w, h


def scales_of(y, block):
    N, d = y.shape
    width = block or d
    most = np.stack([np.max(np.abs(y[:, c:c + width]), axis=1) for c in range(0, d, width)], axis=1)
    return np.maximum(most, LEAST) / E4M3_MAX


def rms_norm_backward(dy, h, w, eps, d_residual=None, mask=None):
    """(dx, dweight, size of dx's terms, size of dweight's terms): the sizes are what errors are measured against."""
    d = h.shape[1]
    h, dy = h.copy(), dy.copy()
    if mask is not None:
        h[mask == 0] = 0.0
        dy[mask == 0] = 0.0
    r = 1.0 / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps)
    u, g = h * r, dy * w
    dx = r * (g - u * np.sum(g * u, axis=1, keepdims=True) / d)
    size = r * (np.abs(g) + np.abs(u) * np.sum(np.abs(g * u), axis=1, keepdims=True) / d)
    if d_residual is not None:
        dx, size = dx + d_residual, size + np.abs(d_residual)
    return dx, np.sum(dy * u, axis=0), size, np.sum(np.abs(dy * u), axis=0)


def grad_norm(grads, max_norm):
    norm = np.sqrt(sum(float(np.sum(g * g)) for g in grads))
    return norm, (min(1.0, max_norm / norm) if norm > 0 else 1.0)


def adamw(p, g, m, v, lr, t, b1=0.9, b2=0.999, eps=1e-8, decay=0.0):
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    return p - lr * (m / (1 - b1 ** t) / (np.sqrt(v / (1 - b2 ** t)) + eps) + decay * p), m, v


def mix(x):
    x = np.asarray(x, dtype=np.uint64)
    low = np.uint64(0xFFFFFFFF)
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x6A09E667)) & low
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0xBB67AE85)) & low
    return x ^ (x >> np.uint64(16))


def random_bits(n, seed, step, place, first=0):
    """The bits of elements first .. first + n - 1."""
    low = np.uint64(0xFFFFFFFF)
    key = mix(place)
    for word in (step & 0xFFFFFFFF, seed >> 32, seed & 0xFFFFFFFF):
        key = mix(np.uint64(word) ^ key)
    i = np.arange(first, first + n, dtype=np.uint64)
    return mix((i & low) ^ mix((key + (i >> np.uint64(32))) & low)).astype(np.int64)


def code_step(x):
    """Distance of the e4m3 values around x >= 0 (the ones above a power of two, at it)."""
    e = np.floor(np.log2(np.maximum(x, 2.0 ** -6)))
    e += (2.0 ** (e + 1) <= x).astype(int) - (2.0 ** e > np.maximum(x, 2.0 ** -6)).astype(int)       # (log2's last bit)
    return 2.0 ** (e - 3)


def to_code(x, u):
    """x in [0, 448] to the e4m3 value below, or above where the fraction and u in [0, 1) reach it."""
    s = code_step(x)
    return np.minimum(np.floor(x / s + u) * s, E4M3_MAX)


def block_max(x, block=256):
    """Largest magnitude of every `block` elements."""
    n = len(x)
    a = np.zeros(-(-n // block) * block)
    a[:n] = np.abs(x)
    return np.maximum(a.reshape(-1, block).max(axis=1), LEAST)


def spread(scale, n, block=256):
    return np.repeat(scale, block)[:n]


def decode(code, scale):
    """Moments from codes (float8 tensor) and scales."""
    return f64(code) * spread(f64(scale), code.numel())


def check_codes(name, got, got_scale, x, bits16, positive, rel=2e-6):
    """Codes and scales of a moment (or square root) x: scales to fp32 rounding, codes those of the oracle wherever x, known to
    `rel`, and the random bits decide."""
    most = block_max(x)
    scale = f64(got_scale)
    # (a maximum of rounded values, a product with 448 and a quotient: each half a step of fp32)
    assert np.all(np.abs(scale - most / E4M3_MAX) <= rel * most / E4M3_MAX), name
    unit = np.abs(x) / spread(most, len(x)) * E4M3_MAX
    u = bits16 / 65536.0
    want = to_code(np.minimum(unit, E4M3_MAX), u)
    if positive:
        want = np.where(x > 0, np.maximum(want, 2.0 ** -9), want)
    q = f64(got)
    z = unit / code_step(unit) + u
    # z is off by at most rel z (z < 17) and a rounding at 2^-20.  A unit that the two sides see on different sides of a power of two, 2^k (1 - e) and 2^k,
    # has z = 16 - 16 e + u and 8 + u there: both mean 2^k but for u < 16 e, where the first z lies at 16.
    open_ = np.abs(z - np.round(z)) < 17 * rel + 2.0 ** -19
    same = np.abs(q) == want
    assert np.all(same | open_), (name, int(np.sum(~(same | open_))))
    # (open ones are 2 (17 rel + 2^-19) = 1.4e-4 of all at most, where zeros with no random bits are not among them: one of a small tensor happens)
    assert np.sum(open_ & (z > 0)) <= 1 + 0.001 * len(x), name
    # (a unit just below a power of two may be seen above it, where steps are twice as long)
    assert np.all(np.abs(np.abs(q) - unit) <= 2.001 * code_step(unit) + (2.0 ** -9 if positive else 0.0)), name
    assert np.all((q == 0) | (np.sign(q) == np.sign(x))), name
