"""What is measured of the operators of a model's fine-tuning: the clipped policy loss and the preference loss with their
gradients, and the orthogonalised update of matrices (by itself and as an optimizer's step), each with its plain form, its
inputs and its definition in 64 bits.

`run` computes the plain form while `own` is false (elementary torch operations in 32 bits, sums over long sequences in 64,
rounded once at the end) and calls the library while it is true.  Widths 64 and 128 and a vocabulary of 256 are those of this
repository's small language model; the other sizes are generic.
"""
import math

import torch

own = False
_ops = None            # the library's module, imported where `own` is true

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
LR, MOMENTUM, DECAY, STEPS, EPS = 0.02, 0.95, 0.1, 5, 1e-7
A, B, C = 3.4445, -4.7750, 2.0315      # x -> A x + B x^3 + C x^5 on singular values
CLIP_LOW, CLIP_HIGH, BETA, SMOOTHING = 0.2, 0.28, 0.1, 0.05


def listed():
    return [
        # the policy loss of the small model's batch: few bytes, where the launch counts
        {"name": "policy small", "op": "policy", "rows": 64, "vocab": 256, "x": "f32", "kl": 0.0, "entropy": 0.01, "masked": 0,
         "idle": 0.0},
        # one optimisation step over sampled answers with a penalty for leaving the reference
        {"name": "policy batch", "op": "policy", "rows": 8192, "vocab": 32000, "x": "bf16", "kl": 0.05, "entropy": 0.0,
         "masked": 0, "idle": 0.0},
        # a padded batch with a large vocabulary, a third of its tokens not answers
        {"name": "policy padded wide", "op": "policy", "rows": 1500, "vocab": 131072, "x": "bf16", "kl": 0.05, "entropy": 0.01,
         "masked": 0, "idle": 0.3},
        # ragged, in 32 bits, odd vocabulary, part of it masked out
        {"name": "policy odd", "op": "policy", "rows": 301, "vocab": 50001, "x": "f32", "kl": 0.1, "entropy": 0.01,
         "masked": 130, "idle": 0.1},
        # a few pairs of short answers
        {"name": "preference few", "op": "preference", "pairs": 8, "tokens": 1999, "weighted": False},
        # a training batch's pairs
        {"name": "preference batch", "op": "preference", "pairs": 256, "tokens": 262144, "weighted": False},
        # the pairs of a whole round of optimisation, weighted
        {"name": "preference large", "op": "preference", "pairs": 4099, "tokens": 12000000, "weighted": True},
        # the small language model's four hidden matrices
        {"name": "muon small", "op": "muon", "dim": 64, "hidden": 128, "layers": 2, "square": False, "p": "f32", "g": "f32"},
        # the hidden matrices of a transformer's blocks, all in 32 bits
        {"name": "muon blocks f32", "op": "muon", "dim": 768, "hidden": 2048, "layers": 8, "square": True, "p": "f32",
         "g": "f32"},
        # larger blocks in 16 bits
        {"name": "muon blocks bf16", "op": "muon", "dim": 2048, "hidden": 5632, "layers": 2, "square": True, "p": "bf16",
         "g": "bf16"},
        # one gradient of odd size in 16 bits
        {"name": "orthogonalize odd f16", "op": "ortho", "batch": 1, "rows": 1001, "cols": 1543, "x": "f16"},
        # a batch of experts' gradients
        {"name": "orthogonalize experts", "op": "ortho", "batch": 8, "rows": 1024, "cols": 2816, "x": "bf16"},
    ]


def _log_uniform(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    n = n if rng.random() < 0.5 else max(lo, n // 64 * 64)     # odd sizes and round ones
    return min(max(n, lo), hi)


def draw(rng):
    op = rng.choice(["policy", "policy", "preference", "muon", "ortho"])
    if op == "policy":
        vocab = _log_uniform(rng, 200, 200000)
        rows = _log_uniform(rng, 1, max(1, min(8192, (1 << 26) // vocab)))
        return {"op": op, "rows": rows, "vocab": vocab, "x": rng.choice(["f32", "bf16", "f16"]), "kl": rng.choice([0.0, 0.05]),
                "entropy": rng.choice([0.0, 0.01]), "masked": rng.choice([0, vocab // 50]), "idle": rng.choice([0.0, 0.25])}
    if op == "preference":
        pairs = _log_uniform(rng, 1, 4096)
        return {"op": op, "pairs": pairs, "tokens": _log_uniform(rng, max(64, 2 * pairs), 8000000),
                "weighted": rng.random() < 0.5}
    if op == "muon":
        dim = _log_uniform(rng, 48, 1600)
        p = rng.choice(["f32", "bf16"])
        return {"op": op, "dim": dim, "hidden": _log_uniform(rng, 48, 2800), "layers": rng.randint(1, 4),
                "square": rng.random() < 0.5, "p": p, "g": rng.choice([p, "f32"])}
    return {"op": op, "batch": rng.choice([1, 1, 3]), "rows": _log_uniform(rng, 32, 2000), "cols": _log_uniform(rng, 32, 2800),
            "x": rng.choice(["bf16", "f16"])}


def _matrices(case):
    """(how many, rows, cols) of each shape"""
    if case["op"] == "ortho":
        return [(case["batch"], case["rows"], case["cols"])]
    d, h, n = case["dim"], case["hidden"], case["layers"]
    return [(n, d, h), (n, h, d)] + ([(n, d, d)] if case["square"] else [])


def work(case):
    op = case["op"]
    if op == "policy":
        rows, v, ex = case["rows"], case["vocab"], BYTES[case["x"]]
        live = rows - int(rows * case["idle"])           # a token of no weight is not read
        return {"bytes": (rows + live) * v * ex + rows * 48, "flops": 14 * live * v}
    if op == "preference":
        return {"bytes": 12 * case["tokens"] + 28 * case["pairs"], "flops": 4 * case["tokens"]}
    # of the two symmetric products only one half is needed
    flops = bytes_ = 0
    for n, r, c in _matrices(case):
        lo, hi = min(r, c), max(r, c)
        flops += n * STEPS * (3 * lo * lo * hi + lo * lo * lo)
        each = 2 * BYTES[case["x"]] if op == "ortho" else 2 * BYTES[case["p"]] + BYTES[case["g"]] + 8
        bytes_ += n * r * c * each
    return {"bytes": bytes_, "flops": flops}


def _library():
    global _ops
    if _ops is None:
        from paper_1903_04488_b200 import train_ops
        _ops = train_ops
    return _ops


# ---- inputs ------------------------------------------------------------------------------------------


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    unit = lambda *s: torch.rand(*s, generator=gen, device="cuda")  # noqa: E731
    return {"policy": _prepare_policy, "preference": _prepare_preference, "muon": _prepare_muon,
            "ortho": _prepare_ortho}[case["op"]](dict(case), gen, rand, unit)


def _prepare_policy(st, gen, rand, unit):
    rows, v = st["rows"], st["vocab"]
    st["ids"] = torch.randint(0, v - st["masked"], (rows,), generator=gen, device="cuda")
    z = rand(rows, v).mul_(2.0)
    z.scatter_add_(1, st["ids"][:, None], 3 * rand(rows, 1) + 6)          # sampled tokens are likely ones
    if st["masked"]:
        z[:, v - st["masked"]:] = -math.inf                               # the padding of the vocabulary
    st["z"] = z.to(DTYPES[st["x"]])
    del z
    zf = st["z"].float()
    logp = zf.gather(1, st["ids"][:, None]).squeeze(1) - zf.logsumexp(-1)
    del zf
    # the policy has moved since it sampled; no ratio within 1e-3 of a border, where either side would be right
    moved = 0.2 * rand(rows)
    for border in (math.log(1 - CLIP_LOW), math.log(1 + CLIP_HIGH)):
        moved = torch.where((moved - border).abs() < 1e-3, moved + 3e-3, moved)
    st["old"] = logp - moved
    st["ref"] = logp + 0.5 * rand(rows) if st["kl"] else None
    st["adv"] = rand(rows)
    w = torch.ones(rows, device="cuda")
    idle = int(rows * st["idle"])
    if idle:
        w[torch.randperm(rows, generator=gen, device="cuda")[:idle]] = 0
    st["w"] = w / w.sum()
    return st


def _prepare_preference(st, gen, rand, unit):
    n, pairs = st["tokens"], st["pairs"]
    # answers of all lengths, some of none, and padding behind the last
    cuts = torch.randint(0, n - n // 50 + 1, (2 * pairs - 1,), generator=gen, device="cuda").sort().values
    ends = torch.tensor([0, n - n // 50], device="cuda")
    st["starts"] = torch.cat([ends[:1], cuts, ends[1:]]).to(torch.int32)
    st["logp"] = torch.log(unit(n).clamp_min(1e-6))
    st["ref"] = st["logp"] + 0.05 * rand(n)
    st["w"] = unit(pairs) / pairs if st["weighted"] else None
    return st


def _gradients(rand, shape):
    """A few strong directions over noise, as gradients of matrices have."""
    n, r, c = shape
    k = max(1, min(r, c) // 32)
    return 0.02 * (rand(n, r, k) @ rand(n, k, c) / math.sqrt(k) + rand(n, r, c)) * torch.exp(rand(n, 1, c))


def _prepare_ortho(st, gen, rand, unit):
    x = _gradients(rand, _matrices(st)[0]).to(DTYPES[st["x"]])
    st["data"] = x if st["batch"] > 1 else x[0]
    return st


def _prepare_muon(st, gen, rand, unit):
    shapes = _matrices(st)
    # one flat vector each, the matrices of a shape side by side
    st["p"] = torch.cat([(rand(n, r, c) / math.sqrt(c)).view(-1) for n, r, c in shapes]).to(DTYPES[st["p"]])
    st["g"] = torch.cat([_gradients(rand, s).view(-1) for s in shapes]).to(DTYPES[st["g"]])
    st["m"] = torch.cat([_gradients(rand, s).view(-1) for s in shapes])
    sizes = [n * r * c for n, r, c in shapes]
    st["stacks"] = list(zip(*[[piece.view(s) for piece, s in zip(st[k].split(sizes), shapes)] for k in ("p", "g", "m")]))
    if own:
        # the handle that a program keeps
        cut = lambda k: [t for stack in st["stacks"] for t in stack[k]]  # noqa: E731
        st["grads"] = cut(1)
        st["opt"] = _library().Muon(cut(0), lr=LR, momentum=MOMENTUM, weight_decay=DECAY, steps=STEPS, coefficients=(A, B, C),
                                    eps=EPS, scale="rms", m=cut(2))
    return st


# ---- one pass ----------------------------------------------------------------------------------------


def run(st):
    return (_run_own if own else _run_plain)(st)


def _run_own(st):
    train_ops = _ops or _library()
    op = st["op"]
    if op == "policy":
        r = train_ops.policy_loss(st["z"], st["ids"], st["old"], st["adv"], ref_logp=st["ref"], weights=st["w"],
                                  clip=(CLIP_LOW, CLIP_HIGH), kl=st["kl"], entropy=st["entropy"])
        return {"stats": r.stats, "dlogits": r.dlogits}
    if op == "preference":
        r = train_ops.preference_loss(st["logp"], st["ref"], st["starts"], beta=BETA, label_smoothing=SMOOTHING, weights=st["w"])
        return {"loss": r.loss, "rewards": r.rewards, "d_logp": r.d_logp}
    if op == "ortho":
        return train_ops.orthogonalize(st["data"], steps=STEPS, coefficients=(A, B, C), eps=EPS)
    st["opt"].step(st["grads"])
    return {"p": st["p"], "m": st["m"]}


def _run_plain(st):
    return {"policy": _policy, "preference": _preference, "muon": _muon, "ortho": _ortho}[st["op"]](st)


def _policy(st):
    z, w = st["z"].float(), st["w"]
    top = z.amax(-1, keepdim=True)
    d = z - top
    e = torch.exp(d)
    s = e.sum(-1, keepdim=True)
    logp = d - torch.log(s)                                  # of every token
    p = e / s
    h = -torch.where(p > 0, p * logp, 0.0).sum(-1)
    at = logp.gather(1, st["ids"][:, None]).squeeze(1)
    ratio = torch.exp(at - st["old"])
    adv = st["adv"]
    kept = torch.where(adv >= 0, ratio.clamp_max(1 + CLIP_HIGH), ratio.clamp_min(1 - CLIP_LOW))
    loss = -kept * adv - st["entropy"] * h
    c = torch.where(kept == ratio, -adv * ratio, 0.0)
    kl = torch.zeros_like(at)
    if st["ref"] is not None:
        q = st["ref"] - at
        kl = torch.expm1(q) - q
        loss = loss + st["kl"] * kl
        c = c - st["kl"] * torch.expm1(q)
    dz = -p * c[:, None]
    if st["entropy"]:
        dz = dz + torch.where(p > 0, p * (logp + h[:, None]), 0.0) * st["entropy"]
    dz.scatter_add_(1, st["ids"][:, None], c[:, None])
    live = w != 0                                            # a token of no weight has no statistics either
    stats = torch.where(live, torch.stack([w * loss, at, h, kl, ratio]), 0.0)
    return {"stats": stats, "dlogits": torch.where(live[:, None], dz * w[:, None], 0.0).to(st["z"].dtype)}


def _preference(st):
    starts = st["starts"].long()
    total = torch.cumsum(st["logp"].double() - st["ref"].double(), 0)
    upto = torch.where(starts > 0, total[(starts - 1).clamp_min(0)], 0.0)
    delta = (upto[1:] - upto[:-1]).float().view(-1, 2)
    x = BETA * (delta[:, 0] - delta[:, 1])
    # -log sigmoid(x) = max(-x, 0) + log(1 + e^-|x|)
    soft = torch.log1p(torch.exp(-x.abs()))
    lose = 1 / (1 + torch.exp(x))                            # sigmoid(-x)
    w = 1.0 if st["w"] is None else st["w"]
    loss = w * ((1 - SMOOTHING) * ((-x).clamp_min(0) + soft) + SMOOTHING * (x.clamp_min(0) + soft))
    slope = w * BETA * (SMOOTHING - lose)
    # a token's sequence: how many starts are at or before it
    seq = torch.bucketize(torch.arange(st["tokens"], device="cuda"), starts, right=True) - 1
    each = torch.cat([torch.stack([slope, -slope], 1).view(-1), slope.new_zeros(1)])
    return {"loss": loss, "rewards": BETA * delta.t().contiguous(), "d_logp": each[seq]}


def _iterate(x):
    """STEPS times x -> A x + (B x x' + C (x x')^2) x, over the shorter side."""
    tall = x.shape[-2] > x.shape[-1]
    x = x.mT if tall else x
    x = x / ((x * x).sum((-2, -1), keepdim=True).sqrt() + EPS)
    for _ in range(STEPS):
        g = x @ x.mT
        x = A * x + (B * g + C * (g @ g)) @ x
    return x.mT if tall else x


def _ortho(st):
    return _iterate(st["data"].float()).to(st["data"].dtype).contiguous()


def _muon(st):
    for p, g, m in st["stacks"]:
        g = g.float()
        m.copy_(m * MOMENTUM + g * (1 - MOMENTUM))
        update = _iterate(m * MOMENTUM + g * (1 - MOMENTUM))
        scale = 0.2 * math.sqrt(max(p.shape[-2:]))
        p.copy_(p.float() * (1 - LR * DECAY) - (LR * scale) * update)
    return {"p": st["p"], "m": st["m"]}


# ---- the definitions in 64 bits ----------------------------------------------------------------------


def exact(case, seed):
    global own
    mine, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = mine
    return {"policy": _exact_policy, "preference": _exact_preference, "muon": _exact_muon, "ortho": _exact_ortho}[case["op"]](st)


def _exact_policy(st):
    rows = torch.arange(st["rows"], device="cuda")
    f = lambda k: st[k].to(torch.float64)  # noqa: E731
    logp = torch.log_softmax(f("z"), -1)
    at = logp[rows, st["ids"]].clone()
    h = -torch.special.xlogy(logp.exp(), logp.exp()).sum(-1)
    rho = (at - f("old")).exp()
    lo, hi = 1 - CLIP_LOW, 1 + CLIP_HIGH
    a, b = rho * f("adv"), rho.clamp(lo, hi) * f("adv")
    loss = -torch.minimum(a, b) - st["entropy"] * h
    # the slope along log p of the sampled token
    along = -torch.where(a <= b, a, torch.zeros_like(a))
    kl = torch.zeros_like(at)
    if st["ref"] is not None:
        u = (f("ref") - at).exp()
        kl = u - 1 - u.log()
        loss, along = loss + st["kl"] * kl, along + st["kl"] * (1 - u)
    w = f("w")
    # d log p_id / d z_j = [j = id] - p_j and d H / d z_j = -p_j (log p_j + H)
    dz = torch.special.xlogy(logp.exp(), logp.exp()).add_(logp.exp() * h[:, None]).mul_(st["entropy"])
    dz -= logp.exp() * along[:, None]
    dz[rows, st["ids"]] += along
    dz *= w[:, None]
    gone = w == 0
    dz[gone] = 0
    stats = torch.stack([w * loss, at, h, kl, rho])
    stats[:, gone] = 0
    return {"stats": stats, "dlogits": dz}


def _exact_preference(st):
    n, pairs = st["tokens"], st["pairs"]
    lens = st["starts"].long().diff()
    seq = torch.repeat_interleave(torch.arange(2 * pairs, device="cuda"), lens)
    diff = (st["logp"].double() - st["ref"].double())[: seq.numel()]
    delta = torch.zeros(2 * pairs, dtype=torch.float64, device="cuda").index_add_(0, seq, diff)
    x = BETA * (delta[0::2] - delta[1::2])
    w = torch.ones_like(x) if st["w"] is None else st["w"].double()
    loss = -w * ((1 - SMOOTHING) * torch.nn.functional.logsigmoid(x) + SMOOTHING * torch.nn.functional.logsigmoid(-x))
    # d/dx of the bracket: (1 - s) sigmoid(-x) - s sigmoid(x)
    slope = -w * BETA * ((1 - SMOOTHING) * torch.sigmoid(-x) - SMOOTHING * torch.sigmoid(x))
    d = torch.zeros(n, dtype=torch.float64, device="cuda")
    d[: seq.numel()] = torch.stack([slope, -slope], 1).flatten()[seq]
    return {"loss": loss, "rewards": BETA * torch.stack([delta[0::2], delta[1::2]]), "d_logp": d}


def _exact_iterate(x):
    # x_k = q_k(G) x_0 with G = x_0 x_0': the polynomials of G commute, so only G's are multiplied
    wide = x if x.shape[-2] <= x.shape[-1] else x.transpose(-1, -2)
    unit = 1 / (torch.linalg.vector_norm(wide, dim=(-2, -1), keepdim=True) + EPS)
    gram = torch.matmul(wide, wide.transpose(-1, -2)) * unit * unit
    eye = torch.eye(wide.shape[-2], dtype=torch.float64, device=x.device).expand_as(gram)
    total = eye
    for _ in range(STEPS):
        q = A * eye + torch.matmul(gram, B * eye + C * gram)
        total = torch.matmul(q, total)
        gram = torch.matmul(torch.matmul(q, gram), q)
    y = torch.matmul(total, wide) * unit
    return y if wide is x else y.transpose(-1, -2)


def _exact_ortho(st):
    return _exact_iterate(st["data"].double()).contiguous()


def _exact_muon(st):
    ps, ms = [], []
    for p, g, m in st["stacks"]:
        p, g, m = p.double(), g.double(), m.double()
        m = MOMENTUM * m + (1 - MOMENTUM) * g
        step = _exact_iterate(MOMENTUM * m + (1 - MOMENTUM) * g) * (0.2 * math.sqrt(max(p.shape[1], p.shape[2])))
        ps.append((p - LR * (DECAY * p + step)).reshape(-1))
        ms.append(m.reshape(-1))
    return {"p": torch.cat(ps), "m": torch.cat(ms)}
