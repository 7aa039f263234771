"""Performance cases of what a step needs that learns from a teacher's distribution: the top alternatives of given logits with the
log-probs of given tokens and the entropy, the distillation loss on a teacher's top log-probs through the head (forward and backward), and the
embedding lookup with its gradient.

Plain forms in elementary torch operations stand beside the calls of the library.  Widths and vocabularies are those of the benchmark
configurations (d = 1536, 2048, 3584, 4096; V = 128256, 151936) and odd ones."""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # the answer of one decoding step of one sequence: log-prob of the sampled token, entropy, eight alternatives; all latency
        dict(name="top_token", call="top", N=1, V=151936, pad=0, k=8, z="f32", T=1.0, scored=1.0),
        # a decoding step of 48 sequences whose logits come with padded rows
        dict(name="top_batch", call="top", N=48, V=128256, pad=192, k=20, z="f32", T=1.0, scored=1.0),
        # odd everything: a smaller vocabulary, rows that begin anywhere, some of them not wanted, softened
        dict(name="top_odd", call="top", N=777, V=50257, pad=0, k=33, z="f32", T=2.0, scored=0.8),
        # a teacher's logits of a micro-batch become targets of 64 alternatives
        dict(name="top_teacher", call="top", N=4096, V=151936, pad=0, k=64, z="bf16", T=1.0, scored=1.0),
        # a gradient check's size, all in 32 bits
        dict(name="distill_tiny", call="distill", N=256, d=64, V=512, k=16, h="f32", T=1.0, renormalize=1, weights=0, scored=0.9),
        # a few short answers through a large head
        dict(name="distill_short", call="distill", N=200, d=1536, V=151936, k=32, h="bf16", T=1.0, renormalize=1, weights=0, scored=1.0),
        # odd width and vocabulary, softened, weighted rows, truncated probabilities, padded batch
        dict(name="distill_odd", call="distill", N=1500, d=712, V=50257, k=50, h="bf16", T=2.0, renormalize=0, weights=1, scored=0.6),
        # a micro-batch of long answers through the largest head
        dict(name="distill_large", call="distill", N=8192, d=4096, V=151936, k=64, h="bf16", T=1.0, renormalize=1, weights=1, scored=1.0),
        # the next tokens of 32 sequences
        dict(name="embed_tokens", call="embed", N=32, d=4096, V=151936, e="bf16", y="bf16", scale=1.0, scored=1.0),
        # prompts of a whole batch, scaled by the root of the width
        dict(name="embed_prompt", call="embed", N=32768, d=3584, V=151936, e="bf16", y="bf16", scale=3584.0 ** 0.5, scored=1.0),
        # gradient of a small table, odd width, padded batch, all in 32 bits
        dict(name="embed_back_odd", call="embed_back", N=3001, d=713, V=32000, y="f32", e="f32", scale=713.0 ** 0.5, scored=0.7),
        # gradient of the largest table from a whole micro-batch, whose most common token is a twentieth of it
        dict(name="embed_back_large", call="embed_back", N=65536, d=4096, V=151936, y="bf16", e="f32", scale=1.0, scored=1.0),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    call = rng.choice(["top", "top", "distill", "distill", "distill", "embed", "embed_back", "embed_back"])
    scored = rng.choice([1.0, 1.0, 0.34, rng.uniform(0.05, 1.0)])
    V = rng.choice([151936, 128256, 50257, log_int(300, 151936), log_int(300, 151936)])
    if call == "top":
        N = log_int(1, 16384)
        while N * V > 4096 * 151936:
            N = max(1, N // 3)
        return dict(call=call, N=N, V=V, pad=rng.choice([0, 0, rng.randint(1, 300)]), k=log_int(1, 200), z=rng.choice(["f32", "bf16"]),
                    T=rng.choice([1.0, 1.0, 2.0, rng.uniform(0.5, 4.0)]), scored=scored)
    if call == "distill":
        h = rng.choice(["bf16", "bf16", "bf16", "f32"])
        if h == "f32":
            N, d, V = log_int(1, 2048), log_int(8, 256), log_int(300, 4000)
        else:
            N, d = log_int(1, 16384), rng.choice([1536, 2048, 3584, 4096, 8 * log_int(8, 512)])
            while N * d * V > 8192 * 4096 * 151936:
                N = max(1, N // 3)
        return dict(call=call, N=N, d=d, V=V, k=log_int(1, 200), h=h, T=rng.choice([1.0, 1.0, 2.0, rng.uniform(0.7, 4.0)]),
                    renormalize=rng.randint(0, 1), weights=rng.randint(0, 1), scored=scored)
    d = rng.choice([1536, 2048, 3584, 4096, log_int(16, 8192), 8 * log_int(8, 1024)])
    e = rng.choice(["bf16", "bf16", "f32"])
    while V * d > 151936 * 4096:
        V = V // 2
    N = log_int(1, 65536)
    while N * d > 65536 * 4096:
        N = N // 2
    return dict(call=call, N=N, d=d, V=V, y=rng.choice(["bf16", "f32"]), e=e, scale=rng.choice([1.0, d ** 0.5]), scored=scored)


# ------------------------------------------------------------------------------------------ inputs
def _scored(c):
    return c["N"] if c["scored"] == 1.0 else max(1, round(c["scored"] * c["N"]))


def prepare(case, seed):
    c = case
    N, V = c["N"], c["V"]
    g = torch.Generator(DEV).manual_seed(seed)

    def normal(*shape, dtype=torch.float32):
        return torch.randn(shape, device=DEV, generator=g, dtype=dtype)

    s = dict(case=c)
    # (exactly as many scored rows for every seed)
    s["mask"] = None if c["scored"] == 1.0 else (torch.randperm(N, device=DEV, generator=g) < _scored(c)).to(torch.uint8)
    if c["call"] == "top":
        z = normal(N, V + c["pad"], dtype=TYPES[c["z"]])
        z *= 1.5 + 2.5 * torch.rand(N, 1, device=DEV, generator=g).to(z.dtype)           # some rows are surer than others
        s["z"] = z[:, :V]
        s["targets"] = torch.randint(0, V, (N,), device=DEV, generator=g, dtype=torch.int32)
        return s
    if c["call"] == "distill":
        d, dtype = c["d"], TYPES[c["h"]]
        s["h"] = normal(N, d).to(dtype)
        s["w"] = normal(V, d).mul_(3.0 / d ** 0.5).to(dtype)
        # a teacher that the student resembles: its alternatives, best first, with their log-probs at the temperature; now and then fewer of them
        teacher = (0.8 * s["h"].float() + 0.6 * normal(N, d)).to(dtype)
        ids = torch.empty(N, c["k"], device=DEV, dtype=torch.int32)
        logp = torch.empty(N, c["k"], device=DEV)
        for at in range(0, N, 2048):
            z = (teacher[at:at + 2048] @ s["w"].t()).float() / c["T"]
            top, best = z.topk(c["k"], dim=1)
            ids[at:at + 2048] = best
            logp[at:at + 2048] = top - z.logsumexp(1, keepdim=True)
        short = (torch.rand(N, 1, device=DEV, generator=g) < 0.2) & (torch.arange(c["k"], device=DEV) >= max(1, c["k"] // 2))
        s["ids"], s["logp"] = torch.where(short, -1, ids), logp
        s["weight"] = torch.rand(N, device=DEV, generator=g).add_(0.5).div_(N) if c["weights"] else None
        return s
    # token ids as texts have them: the i-th most common one about 1 / i as often as the first, numbered in no order
    u = torch.rand(N, device=DEV, generator=g, dtype=torch.float64)
    rank = torch.exp(u * math.log(V)).long().sub_(1).clamp_(0, V - 1)
    s["ids"] = torch.randperm(V, device=DEV, generator=g)[rank].to(torch.int32)
    if c["call"] == "embed":
        s["table"] = normal(V, c["d"]).mul_(0.02).to(TYPES[c["e"]])
    else:
        s["dy"] = normal(N, c["d"]).mul_(0.01 * torch.exp(normal(N, 1))).to(TYPES[c["y"]])
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["case"]
    if own:
        import paper_2605_07244_amd as mrl
    if c["call"] == "top":
        if own:
            r = mrl.top_logprobs(s["z"], c["k"], target_ids=s["targets"], token_mask=s["mask"], temperature=c["T"])
            return dict(ids=r["ids"], top=r["top_logp"], logp=r["logp"], lse=r["lse"], entropy=r["entropy"])
        return _top(s["z"], c["k"], s["targets"], s["mask"], c["T"])
    if c["call"] == "distill":
        if own:
            cfg = mrl.DistillConfig(temperature=c["T"], renormalize=c["renormalize"], dh_dtype=mrl.BF16 if c["h"] == "bf16" else mrl.F32,
                                    dw_dtype=mrl.BF16 if c["h"] == "bf16" else mrl.F32)
            r = mrl.distill_loss_fwd_bwd(s["h"], s["w"], s["ids"], s["logp"], cfg, token_mask=s["mask"], row_weight=s["weight"])
            return dict(kl=r["kl"], dH=r["dH"], dW=r["dW"])
        return _distill(s["h"], s["w"], s["ids"], s["logp"], s["mask"], s["weight"], c["T"], c["renormalize"])
    if c["call"] == "embed":
        if own:
            return mrl.embedding(s["table"], s["ids"], scale=c["scale"], token_mask=s["mask"], out_dtype=TYPES[c["y"]])
        y = s["table"].index_select(0, s["ids"]).float() * c["scale"]
        if s["mask"] is not None:
            y = torch.where(s["mask"][:, None] != 0, y, 0.0)
        return y.to(TYPES[c["y"]])
    if own:
        return mrl.embedding_backward(s["dy"], s["ids"], c["V"], scale=c["scale"], token_mask=s["mask"], out_dtype=TYPES[c["e"]])
    dy = s["dy"].float()
    if s["mask"] is not None:
        dy = torch.where(s["mask"][:, None] != 0, dy, 0.0)
    table = torch.zeros(c["V"], c["d"], device=DEV).index_add_(0, s["ids"], dy)
    return table.mul_(c["scale"]).to(TYPES[c["e"]])


def _unique(c):
    """How many tokens of the table occur among N, on average."""
    i = torch.arange(1, c["V"] + 1, dtype=torch.float64)
    p = torch.log1p(1 / i) / math.log(c["V"] + 1)
    return float((1 - (1 - p) ** _scored(c)).sum())


def work(case):
    c = case
    N, V, n = c["N"], c["V"], _scored(c)
    size = lambda t: {"f32": 4, "bf16": 2}[t]
    mask = 0 if c["scored"] == 1.0 else N
    if c["call"] == "top":
        return {"bytes": n * V * size(c["z"]) + N * (8 * c["k"] + 16) + mask, "flops": 5 * n * V}
    if c["call"] == "distill":
        d, e = c["d"], size(c["h"])
        return {"bytes": (n + N) * d * e + 2 * V * d * e + 8 * n * c["k"] + 4 * N * (1 + c["weights"]) + mask, "flops": 6 * n * d * V}
    d = c["d"]
    if c["call"] == "embed":
        return {"bytes": _unique(c) * d * size(c["e"]) + N * d * size(c["y"]) + 4 * N + mask, "flops": n * d}
    return {"bytes": n * d * size(c["y"]) + V * d * size(c["e"]) + 4 * N + mask, "flops": n * d}


# ------------------------------------------------------------------------------------------ plain forms
def _top(z, k, targets, mask, T):
    s = z.float() / T
    biggest = s.amax(1, keepdim=True)
    e = torch.exp(s - biggest)
    total = e.sum(1, keepdim=True)
    lse = biggest + torch.log(total)
    p = e / total
    entropy = lse[:, 0] - (p * s).sum(1)
    logp = s.gather(1, targets.long()[:, None])[:, 0] - lse[:, 0]
    values, order = torch.sort(z, dim=1, descending=True, stable=True)
    ids = order[:, :k].to(torch.int32)
    top = values[:, :k].float() / T - lse
    lse = lse[:, 0]
    if mask is not None:
        on = mask != 0
        lse, entropy, logp = (torch.where(on, x, 0.0) for x in (lse, entropy, logp))
        ids, top = torch.where(on[:, None], ids, -1), torch.where(on[:, None], top, 0.0)
    return dict(ids=ids, top=top, logp=logp, lse=lse, entropy=entropy)


def _distill(h, w, ids, logp, mask, weight, T, renormalize):
    h32, w32 = h.float(), w.float()
    there = ids >= 0
    on = there.any(1) if mask is None else there.any(1) & (mask != 0)
    best = torch.where(there, logp, -math.inf).amax(1, keepdim=True)
    q = torch.where(there, torch.exp(logp - best), 0.0)
    q = q / q.sum(1, keepdim=True) if renormalize else q * torch.exp(best)
    log_q = torch.log(torch.where(q > 0, q, 1.0))
    s = (h32 @ w32.t()) / T
    s = s - s.amax(1, keepdim=True)
    e = torch.exp(s)
    total = e.sum(1, keepdim=True)
    at = ids.clamp(min=0).long()
    log_p = s.gather(1, at) - torch.log(total)
    kl = torch.where(on, (q * (log_q - log_p)).sum(1), 0.0)
    c = torch.where(on, weight if weight is not None else 1.0 / on.sum(), 0.0) * T
    dz = e.mul_(q.sum(1, keepdim=True) / total).scatter_add_(1, at, -q).mul_(c[:, None])
    return dict(kl=kl, dH=(dz @ w32).to(h.dtype), dW=(dz.t() @ h32).to(w.dtype))


# ------------------------------------------------------------------------------------------ in 64 bits
def _ordered(z):
    """Whole numbers in the order of the values, zeros of either sign alike."""
    bits = (z.float() + 0.0).view(torch.int32).long()
    return torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)


def _exact_top(s, c):
    parts = []
    for at in range(0, c["N"], 512):
        z = s["z"][at:at + 512]
        keys = _ordered(z) * 2 ** 24 + (2 ** 24 - 1 - torch.arange(c["V"], device=DEV))       # (no two alike: the lower id is the larger one)
        ids = 2 ** 24 - 1 - keys.topk(c["k"], dim=1, sorted=True).values % 2 ** 24
        x = z.double() / c["T"]
        lse = torch.logsumexp(x, 1)
        logs = x - lse[:, None]
        target = s["targets"][at:at + 512].long()[:, None]
        parts.append(dict(ids=ids.to(torch.int32), top=torch.take_along_dim(logs, ids, 1), logp=torch.take_along_dim(logs, target, 1)[:, 0], lse=lse,
                          entropy=-(torch.exp(logs) * logs).sum(1)))
    out = {name: torch.cat([p[name] for p in parts]) for name in parts[0]}
    if s["mask"] is not None:
        off = s["mask"] == 0
        for name, x in out.items():
            x[off] = -1 if name == "ids" else 0
    return out


def _exact_distill(s, c):
    h, w, T = s["h"].double(), s["w"].double(), c["T"]
    N, V = c["N"], c["V"]
    on = (s["ids"] >= 0).sum(1) > 0
    if s["mask"] is not None:
        on &= s["mask"] != 0
    rows = on.nonzero()[:, 0]
    weight = s["weight"].double() if s["weight"] is not None else torch.full((N,), 1.0 / len(rows), device=DEV, dtype=torch.float64)
    kl = torch.zeros(N, device=DEV, dtype=torch.float64)
    dH, dW = torch.zeros_like(h), torch.zeros_like(w)
    for part in rows.split(2048):
        log_p = torch.log_softmax(h[part] @ w.t() / T, 1)
        ids, t = s["ids"][part], s["logp"][part].double()
        t = t.masked_fill(ids < 0, -math.inf)
        q = torch.softmax(t, 1) if c["renormalize"] else torch.exp(t)
        index = ids.clamp(min=0).long()
        kl[part] = (torch.special.xlogy(q, q) - q * torch.take_along_dim(log_p, index, 1)).sum(1)
        dz = log_p.exp_() * q.sum(1)[:, None]
        dz -= torch.zeros_like(dz).scatter_add_(1, index, q)
        dz *= (weight[part] * T)[:, None]
        dH[part] = dz @ w
        dW += dz.t() @ h[part]
    return dict(kl=kl, dH=dH, dW=dW)


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["call"] == "top":
        return _exact_top(s, c)
    if c["call"] == "distill":
        return _exact_distill(s, c)
    on = torch.ones(c["N"], device=DEV, dtype=torch.bool) if s["mask"] is None else s["mask"] != 0
    ids = s["ids"].long()
    if c["call"] == "embed":
        return s["table"].double()[ids] * (on * c["scale"])[:, None]
    out = torch.zeros(c["V"], c["d"], device=DEV, dtype=torch.float64)
    out.index_put_((ids[on],), s["dy"][on].double() * c["scale"], accumulate=True)
    return out
