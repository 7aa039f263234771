"""Performance cases of the operators around the scoring step: the final norm in front of it (forward, with the residual's
addition and outputs in 32, 16 or 8 bits) and behind it (backward), the gradients' global norm, and the AdamW update.

Plain forms in elementary torch operations stand beside the calls of the library.  Widths are those of the benchmark
configurations (1536, 2048, 3584, 4096) and odd ones; heads are theirs too ([V, d] of up to 263 M weights)."""
import math

import torch

own = False

DEV = "cuda"
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
LEAST = 2.0 ** -100            # the least maximum that a scale is made of
STATE_BLOCK = 256              # elements of a tensor that share the scales of 8-bit states
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": E4M3}
BETA1, BETA2, ADAM_EPS = 0.9, 0.999, 1e-8


def listed():
    return [
        # one new token of one sequence passes the norm: all latency
        dict(name="norm_token", call="norm", N=1, d=4096, x="bf16", residual="bf16", w="bf16", y="bf16", block=0, scored=1.0),
        # hidden states for a layer that multiplies 8-bit rows, a prompt's worth of them, a scale per row
        dict(name="norm_e4m3", call="norm", N=2047, d=3584, x="bf16", residual="bf16", w="bf16", y="e4m3", block=0, scored=1.0),
        # final hidden states of a padded micro-batch of 16 x 2048 slots, a third of them scored
        dict(name="norm_masked", call="norm", N=32768, d=4096, x="bf16", residual="bf16", w="f32", y="bf16", block=0, scored=0.34),
        # dH of a few short answers through the norm
        dict(name="back_short", call="back", N=400, d=1536, h="bf16", dy="bf16", residual="bf16", w="bf16", dx="bf16", scored=1.0, accumulate=0),
        # odd everything, in 32 bits, weight gradient accumulated over micro-batches
        dict(name="back_ragged", call="back", N=3001, d=713, h="f32", dy="f32", residual="", w="f32", dx="f32", scored=0.8, accumulate=1),
        # dH of a whole step: 128 rollouts of up to 1024 tokens
        dict(name="back_large", call="back", N=131072, d=2048, h="bf16", dy="bf16", residual="bf16", w="bf16", dx="bf16", scored=0.63, accumulate=0),
        # the norm of many small gradients: norm weights and biases of a whole model
        dict(name="gradnorm_many", call="gradnorm", tensors=57, least=300, most=20000, align=64, grad="f32", max_norm=1.0),
        # the norm of the head's gradient
        dict(name="gradnorm_head", call="gradnorm", tensors=1, least=151936 * 1536, most=151936 * 1536, align=64, grad="f32", max_norm=1.0),
        # clipped update of many small tensors
        dict(name="adamw_many", call="adamw", tensors=57, least=300, most=20000, align=64, grad="f32", states="f32", copy=1, max_norm=1.0,
             lr=3e-4, wd=0.01, step=100),
        # update of the head: float32 gradient, states and weights, the bf16 copy for the next scoring pass
        dict(name="adamw_head", call="adamw", tensors=1, least=151936 * 1536, most=151936 * 1536, align=64, grad="f32", states="f32", copy=1,
             max_norm=0.0, lr=1e-4, wd=0.01, step=1000),
        # matrices of odd sizes one right behind the other in flat buffers, bf16 gradients, states in 8 bits, clipped
        dict(name="adamw8_ragged", call="adamw", tensors=13, least=2000, most=3000000, align=1, grad="bf16", states="e4m3", copy=1, max_norm=1.0,
             lr=3e-4, wd=0.1, step=7),
        # update of a larger head with states in 8 bits
        dict(name="adamw8_head", call="adamw", tensors=1, least=128256 * 2048, most=128256 * 2048, align=64, grad="f32", states="e4m3", copy=1,
             max_norm=0.0, lr=1e-4, wd=0.01, step=1000),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    call = rng.choice(["norm", "norm", "norm", "back", "back", "gradnorm", "adamw", "adamw", "adamw"])
    if call in ("norm", "back"):
        d = rng.choice([1536, 2048, 3584, 4096, log_int(16, 16384), log_int(64, 16384), 8 * log_int(8, 2048)])
        N = log_int(1, 131072)
        while N * d > 131072 * 2048:
            N = max(1, N // 3)
        scored = rng.choice([1.0, 1.0, 0.34, rng.uniform(0.05, 1.0)])
        if call == "norm":
            x = rng.choice(["bf16", "bf16", "f32"])
            y = rng.choice(["bf16", "e4m3", "e4m3", "f32"])
            return dict(call=call, N=N, d=d, x=x, residual=rng.choice(["", x, "f32"]), w=rng.choice(["bf16", "f32"]), y=y,
                        block=rng.choice([0, 128]) if y == "e4m3" else 0, scored=scored)
        h = rng.choice(["bf16", "bf16", "f32"])
        return dict(call=call, N=N, d=d, h=h, dy=rng.choice(["bf16", "f32"]), residual=rng.choice(["", h]), w=rng.choice(["bf16", "f32"]),
                    dx=rng.choice(["bf16", h]), scored=scored, accumulate=rng.randint(0, 1))
    tensors = log_int(1, 150)
    most = log_int(50, 230e6 / tensors)
    c = dict(call=call, tensors=tensors, least=rng.choice([1, most, max(1, most // 3)]), most=most, align=rng.choice([64, 64, 1]),
             grad=rng.choice(["f32", "f32", "bf16"]), max_norm=rng.choice([1.0, rng.uniform(0.1, 10.0)]))
    if call == "adamw":
        c.update(states=rng.choice(["f32", "e4m3"]), copy=rng.randint(0, 1), max_norm=rng.choice([0.0, c["max_norm"]]), lr=rng.choice([1e-6, 1e-4, 1e-3]),
                 wd=rng.choice([0.0, 0.01, 0.1]), step=log_int(1, 20000))
    return c


# ------------------------------------------------------------------------------------------ inputs
def _sizes(c):
    """The tensors' sizes: spread evenly over the logarithm of [least, most], the largest first."""
    n, lo, hi = c["tensors"], math.log(c["least"]), math.log(c["most"])
    return [c["most"] if n == 1 else int(round(math.exp(hi - (hi - lo) * i / (n - 1)))) for i in range(n)]


def _places(sizes, align):
    """Where each tensor begins in a flat buffer, and the buffer's length."""
    at, places = 0, []
    for n in sizes:
        places.append(at)
        at += -(-n // align) * align
    return places, at


def prepare(case, seed):
    c = case
    g = torch.Generator(DEV).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, device=DEV, generator=g)

    if c["call"] in ("norm", "back"):
        N, d = c["N"], c["d"]
        size = torch.exp(0.5 * normal(N, 1))                       # rows differ in size, columns a little
        s = dict(case=c, eps=1e-6, w=(1 + 0.2 * normal(d)).to(TYPES[c["w"]]))
        # (exactly as many scored rows for every seed)
        s["mask"] = None if c["scored"] == 1.0 else (torch.randperm(N, device=DEV, generator=g) < max(1, round(c["scored"] * N))).to(torch.uint8)
        if c["call"] == "norm":
            s["x"] = normal(N, d).mul_(size).to(TYPES[c["x"]])
            s["residual"] = normal(N, d).mul_(3 * size).to(TYPES[c["residual"]]) if c["residual"] else None
        else:
            s["h"] = normal(N, d).mul_(3 * size).to(TYPES[c["h"]])
            s["dy"] = normal(N, d).mul_(0.01 * torch.exp(normal(N, 1))).to(TYPES[c["dy"]])
            s["residual"] = normal(N, d).mul_(0.01).to(TYPES[c["residual"]]) if c["residual"] else None
            s["dw"] = 0.1 * normal(d) if c["accumulate"] else None
        return s

    sizes = _sizes(c)
    places, total = _places(sizes, c["align"])

    def parts(flat, sizes=sizes, places=places):
        return [flat[p:p + n] for p, n in zip(places, sizes)]

    s = dict(case=c, sizes=sizes)
    # gradients whose size differs from place to place, as those of a head's rows do
    sigma = 1e-3 * torch.exp(1.5 * normal(total // 1024 + 1)).repeat_interleave(1024)[:total]
    grads = normal(total).mul_(sigma).to(TYPES[c["grad"]])
    s["grads"] = parts(grads)
    if c["call"] == "gradnorm":
        if own:
            import paper_2605_07244_amd as mrl
            s["plan"] = mrl.grad_plan(s["grads"])
        return s
    s["param"] = normal(total).mul_(0.02)
    s["copy"] = s["param"].to(torch.bfloat16) if c["copy"] else None
    m, root = normal(total).mul_(0.3 * sigma), torch.rand(total, device=DEV, generator=g).add_(0.5).mul_(sigma)     # of a run under way
    if c["states"] == "f32":
        s["m"], s["v"], s["m_scale"], s["v_scale"] = m, root.square_(), None, None
        scales = [None] * len(sizes)
    else:
        blocks = [-(-n // STATE_BLOCK) for n in sizes]
        at, length = _places(blocks, 1)
        s["m"], s["v"] = (torch.zeros(total, device=DEV, dtype=E4M3) for _ in range(2))
        s["m_scale"], s["v_scale"] = (torch.zeros(length, device=DEV) for _ in range(2))
        scales = list(zip(parts(s["m_scale"], blocks, at), parts(s["v_scale"], blocks, at)))
        for x, code, k in ((m, "m", 0), (root, "v", 1)):
            for t, q, sc in zip(parts(x), parts(s[code]), scales):
                sc[k].copy_(_by_block(t.abs()).amax(1).clamp_(min=LEAST) / E4M3_MAX)
                q.copy_((t / sc[k].repeat_interleave(STATE_BLOCK)[:t.numel()]).clamp_(-E4M3_MAX, E4M3_MAX).to(E4M3))
    s["tensors"] = list(zip(parts(s["param"]), parts(s["copy"]) if c["copy"] else [None] * len(sizes), s["grads"], parts(s["m"]), parts(s["v"]), scales))
    if own:
        import paper_2605_07244_amd as mrl
        p, copies, grads, m, v, scales = zip(*s["tensors"])
        s["plan"] = mrl.adamw_plan(p, grads, copies if c["copy"] else None, m=m, v=v, m_scale=[x[0] for x in scales] if scales[0] else None,
                                   v_scale=[x[1] for x in scales] if scales[0] else None, weight_decay=c["wd"])
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["case"]
    if c["call"] == "norm":
        if own:
            import paper_2605_07244_amd as mrl
            y, h, scale = mrl.rms_norm(s["x"], s["w"], s["eps"], residual=s["residual"], token_mask=s["mask"], out_dtype=TYPES[c["y"]], scale_block=c["block"])
        else:
            y, h, scale = _norm(s["x"], s["w"], s["eps"], s["residual"], s["mask"], TYPES[c["y"]], c["block"])
        return dict(y=y) | (dict(h=h) if h is not None else {}) | (dict(scale=scale) if scale is not None else {})
    if c["call"] == "back":
        if own:
            import paper_2605_07244_amd as mrl
            dx, dw = mrl.rms_norm_backward(s["dy"], s["h"], s["w"], s["eps"], d_residual=s["residual"], token_mask=s["mask"], dx_dtype=TYPES[c["dx"]],
                                           out_dweight=s["dw"], accumulate=bool(c["accumulate"]))
        else:
            dx, dw = _norm_backward(s["dy"], s["h"], s["w"], s["eps"], s["residual"], s["mask"], TYPES[c["dx"]], s["dw"])
        return dict(dx=dx, dw=dw)
    if c["call"] == "gradnorm":
        if own:
            import paper_2605_07244_amd as mrl
            return mrl.grad_norm(s["plan"], c["max_norm"])
        return _grad_norm(s["grads"], c["max_norm"])
    norm = None
    if own:
        import paper_2605_07244_amd as mrl
        if c["max_norm"]:
            norm = mrl.grad_norm(s["plan"], c["max_norm"])
        mrl.adamw_step(s["plan"], c["lr"], c["step"], beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, norm_coef=norm, seed=c["step"] + 5)
    else:
        if c["max_norm"]:
            norm = _grad_norm(s["grads"], c["max_norm"])
        _adamw(s["tensors"], c, 1.0 if norm is None else norm[1])
    out = dict(param=s["param"], m=s["m"], v=s["v"])
    for name, x in (("copy", s["copy"]), ("m_scale", s["m_scale"]), ("v_scale", s["v_scale"]), ("norm", norm)):
        if x is not None:
            out[name] = x
    return out


def work(case):
    c = case
    bytes_of = lambda t: {"f32": 4, "bf16": 2, "e4m3": 1, "": 0}[t]
    if c["call"] in ("norm", "back"):
        N, d = c["N"], c["d"]
        n = N if c["scored"] == 1.0 else max(1, round(c["scored"] * N))       # rows that are read
        mask = 0 if c["scored"] == 1.0 else N
        if c["call"] == "norm":
            scales = 4 * N * (-(-d // c["block"]) if c["block"] else 1) if c["y"] == "e4m3" else 0
            return {"bytes": n * d * (bytes_of(c["x"]) + bytes_of(c["residual"])) + N * d * (bytes_of(c["residual"]) + bytes_of(c["y"])) + d * bytes_of(c["w"])
                    + scales + mask, "flops": 6 * n * d}
        return {"bytes": n * d * (bytes_of(c["dy"]) + bytes_of(c["h"])) + N * d * (bytes_of(c["residual"]) + bytes_of(c["dx"])) + d * (bytes_of(c["w"])
                + 4 + 4 * c["accumulate"]) + mask, "flops": 13 * n * d}
    sizes = _sizes(c)
    n, g = sum(sizes), bytes_of(c["grad"])
    if c["call"] == "gradnorm":
        return {"bytes": n * g + 8, "flops": 2 * n}
    blocks = sum(-(-x // STATE_BLOCK) for x in sizes) if c["states"] == "e4m3" else 0
    state = bytes_of(c["states"])
    # (the clip coefficient needs every gradient before the first is used: where it is asked for, gradients that no cache holds are read twice)
    twice = g if c["max_norm"] and n * g > 256e6 else 0
    return {"bytes": n * (g + twice + 8 + 4 * state + 2 * c["copy"]) + 16 * blocks, "flops": n * (18 + (2 if c["max_norm"] else 0))}


# ------------------------------------------------------------------------------------------ plain forms
def _norm(x, w, eps, residual, mask, y_type, block):
    h = x.float()
    if residual is not None:
        h = h + residual.float()
    if mask is not None:
        h = torch.where(mask[:, None] != 0, h, 0.0)
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + eps) * w.float()
    total = h.to(residual.dtype) if residual is not None else None
    if y_type != E4M3:
        return y.to(y_type), total, None
    N, d = y.shape
    width = block or d
    parts = torch.nn.functional.pad(y, (0, -d % width)).view(N, -1, width)
    scale = parts.abs().amax(2).clamp(min=LEAST) / E4M3_MAX
    q = (parts / scale[:, :, None]).view(N, -1)[:, :d].contiguous().to(E4M3)
    return q, total, scale if block else scale[:, 0]


def _norm_backward(dy, h, w, eps, residual, mask, dx_type, dw):
    dy, h = dy.float(), h.float()
    if mask is not None:
        dy, h = torch.where(mask[:, None] != 0, dy, 0.0), torch.where(mask[:, None] != 0, h, 0.0)
    r = torch.rsqrt(h.square().mean(1, keepdim=True) + eps)
    g, unit = dy * w.float(), h * r
    dx = r * (g - unit * (g * unit).mean(1, keepdim=True))
    if residual is not None:
        dx = dx + residual.float()
    new = (dy * unit).sum(0)
    return dx.to(dx_type), new if dw is None else dw.add_(new)


def _grad_norm(grads, max_norm):
    norm = torch.stack([g.double().square().sum() for g in grads]).sum().sqrt()
    return torch.stack([norm, torch.clamp(max_norm / norm, max=1.0)]).float()


def _by_block(x):
    """[blocks, STATE_BLOCK], the last one filled up with zeros."""
    return torch.nn.functional.pad(x, (0, -x.numel() % STATE_BLOCK)).view(-1, STATE_BLOCK)


def _mix(x):
    """32 bits mixed, in int64 tensors or Python numbers."""
    x = ((x ^ (x >> 16)) * 0x6A09E667) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random_bits(n, seed, step, tensor):
    key = _mix((seed & 0xFFFFFFFF) ^ _mix((seed >> 32) ^ _mix((step & 0xFFFFFFFF) ^ _mix(tensor))))
    i = torch.arange(n, device=DEV)
    return _mix((i & 0xFFFFFFFF) ^ _mix((key + (i >> 32)) & 0xFFFFFFFF))


def _round(x, u):
    """Multiples of the e4m3 step at x >= 0, up where the fraction and u in [0, 1) reach the next one."""
    step = (x.view(torch.int32) & 0x7F800000).view(torch.float32).clamp(min=2.0 ** -6) / 8
    return (torch.floor(x / step + u) * step).clamp(max=E4M3_MAX)


def _adamw(tensors, c, coef):
    lr, t = c["lr"], c["step"]
    fix1, fix2 = 1 - BETA1 ** t, 1 - BETA2 ** t
    for i, (p, copy, grad, m_at, v_at, scales) in enumerate(tensors):
        n = p.numel()
        g = grad.float() * coef
        m, v = m_at.float(), v_at.float()
        if scales is not None:
            m = (_by_block(m) * scales[0][:, None]).view(-1)[:n]
            v = (_by_block(v) * scales[1][:, None]).view(-1)[:n].square()
        m = BETA1 * m + (1 - BETA1) * g
        v = BETA2 * v + (1 - BETA2) * g * g
        p.copy_(p * (1 - lr * c["wd"]) - lr / fix1 * m / (torch.sqrt(v / fix2) + ADAM_EPS))
        if copy is not None:
            copy.copy_(p)
        if scales is None:
            m_at.copy_(m)
            v_at.copy_(v)
            continue
        bits = _random_bits(n, c["step"] + 5, t, i)
        # (a positive sqrt(v) keeps a positive code)
        for x, u, at, scale, least in ((m, bits & 0xFFFF, m_at, scales[0], 0.0), (torch.sqrt(v), bits >> 16, v_at, scales[1], 2.0 ** -9)):
            most = _by_block(x.abs()).amax(1).clamp(min=LEAST)
            unit = (_by_block(x) * (E4M3_MAX / most)[:, None]).view(-1)[:n]
            q = torch.where(x != 0, _round(unit.abs(), u.float() * 2.0 ** -16).clamp(min=least), 0.0)
            at.copy_((q * x.sign()).to(E4M3))
            scale.copy_(most / E4M3_MAX)


# ------------------------------------------------------------------------------------------ 64 bits
def _to_e4m3_64(x):
    """Nearest e4m3 value, ties to even, of float64 values up to 448."""
    a = x.abs()
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
    return torch.round(a / step).mul_(step).mul_(x.sign())


def _at_random_64(x, u):
    step = torch.exp2(torch.floor(torch.log2(x.clamp(min=2.0 ** -6))) - 3)
    return (torch.floor(x / step + u) * step).clamp_(max=448.0)


def _hash_64(n, seed, step, tensor):
    """The random bits of elements 0 .. n - 1, by the definition: mix(lo(i) ^ mix(key + hi(i)))."""
    def mix(v):
        v = v ^ (v >> 16)
        v = v * 1779033703 % 4294967296
        v = v ^ (v >> 15)
        v = v * 3144134277 % 4294967296
        return v ^ (v >> 16)
    key = mix(tensor)
    for word in (step % 2 ** 32, seed // 2 ** 32, seed % 2 ** 32):
        key = mix(word ^ key)
    i = torch.arange(n, device=DEV, dtype=torch.int64)
    return mix(i % 2 ** 32 ^ mix((key + i // 2 ** 32) % 2 ** 32))


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["call"] == "norm":
        h = s["x"].double() + (s["residual"].double() if c["residual"] else 0.0)
        if s["mask"] is not None:
            h[s["mask"] == 0] = 0.0
        y = h / torch.sqrt((h * h).sum(1, keepdim=True) / c["d"] + s["eps"]) * s["w"].double()
        out = dict(h=h) if c["residual"] else {}
        if c["y"] != "e4m3":
            return dict(out, y=y)
        width = c["block"] or c["d"]
        scale = torch.stack([part.abs().amax(1) for part in y.split(width, dim=1)], dim=1).clamp_(min=2.0 ** -100) / 448
        y = _to_e4m3_64(y / scale.repeat_interleave(width, dim=1)[:, :c["d"]])
        return dict(out, y=y, scale=scale if c["block"] else scale.reshape(-1))
    if c["call"] == "back":
        scored = torch.ones(c["N"], device=DEV, dtype=torch.float64) if s["mask"] is None else s["mask"].double()
        h, dy, w = s["h"].double(), s["dy"].double() * scored[:, None], s["w"].double()
        inv = 1 / torch.sqrt((h * h).sum(1) / c["d"] + s["eps"])
        dw = (dy * h * inv[:, None]).sum(0)
        along = (dy * w * h).sum(1) / c["d"] * inv ** 3
        dx = dy * w * inv[:, None] - h * along[:, None]
        if c["residual"]:
            dx += s["residual"].double()
        return dict(dx=dx, dw=dw + (s["dw"].double() if c["accumulate"] else 0.0))
    squares = sum(float((g.double() ** 2).sum()) for g in s["grads"])
    coef = min(1.0, c["max_norm"] / math.sqrt(squares)) if c["max_norm"] else 1.0
    both = torch.tensor([math.sqrt(squares), coef], dtype=torch.float64)
    if c["call"] == "gradnorm":
        return both
    out = {k: s[k].double() for k in ("param", "copy", "m", "v", "m_scale", "v_scale") if s[k] is not None}     # (what lies between tensors stays)
    places, _ = _places(s["sizes"], c["align"])
    at = 0
    for i, (n, p0) in enumerate(zip(s["sizes"], places)):
        here, blocks = slice(p0, p0 + n), slice(at, at + -(-n // 256))
        at += -(-n // 256)
        spread = (lambda sc: sc.double().repeat_interleave(256)[:n])
        m, v = s["m"][here].double(), s["v"][here].double()
        if c["states"] == "e4m3":
            m, v = m * spread(s["m_scale"][blocks]), (v * spread(s["v_scale"][blocks])) ** 2
        g = s["grads"][i].double() * coef
        m = m + (g - m) * (1 - BETA1)
        v = v + (g * g - v) * (1 - BETA2)
        p = s["param"][here].double()
        denominator = torch.sqrt(v / (1 - BETA2 ** c["step"])) + ADAM_EPS
        p = p - c["lr"] * (m / (1 - BETA1 ** c["step"]) / denominator + c["wd"] * p)
        out["param"][here] = p
        if c["copy"]:
            out["copy"][here] = p
        if c["states"] == "f32":
            out["m"][here], out["v"][here] = m, v
            continue
        bits = _hash_64(n, c["step"] + 5, c["step"], i)
        for x, u, name, least in ((m, bits % 65536, "m", 0.0), (v.sqrt(), bits // 65536, "v", 2.0 ** -9)):
            most = torch.stack([part.max() for part in x.abs().split(256)]) if n < 25600 else torch.nn.functional.pad(x.abs(), (0, -n % 256)).view(-1, 256).amax(1)
            scale = most.clamp(min=2.0 ** -100) / 448
            q = _at_random_64((x.abs() / spread(scale)), u.double() / 65536)
            out[name][here] = torch.where(x != 0, q.clamp(min=least), 0.0) * x.sign()
            out[name + "_scale"][blocks] = scale
    if c["max_norm"]:
        out["norm"] = both
    return out
