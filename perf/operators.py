"""What is measured of the operators around the compression step: layer norm, the log probabilities of given tokens and
the AdamW step, each with its plain form, its inputs and its definition in 64 bits.

`run` computes the plain form while `own` is false (elementary torch operations in 32 bits, rounded once at the end) and
calls the library while it is true.  Sizes: 11,173,962 parameters in 62 tensors and 90,000,000 parameters are the
workloads of this repository; widths, vocabularies and row counts are generic.
"""
import itertools
import math

import torch

own = False
_ops = None            # the library's module, imported where `own` is true

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "none": 0, "e4m3": 1}
LR, BETA1, BETA2, EPS, DECAY, STEP0 = 1e-3, 0.9, 0.95, 1e-8, 0.1, 100
NORM_EPS = 1e-5
BLOCK = 256            # elements that share a scale in an 8-bit state


def listed():
    return [
        # layer norm of one token: a decoder's step, where the launch counts
        {"name": "norm one token", "op": "norm", "rows": 1, "n": 2048, "x": "bf16", "w": "f32"},
        # a training batch's forward pass
        {"name": "norm batch", "op": "norm", "rows": 16384, "n": 2048, "x": "bf16", "w": "bf16"},
        # the same layer's backward pass at a larger width, the weight's gradient reduced over all rows
        {"name": "norm backward", "op": "norm_back", "rows": 16384, "n": 4096, "x": "bf16", "w": "f32"},
        # a small ragged batch of a width that no vector of 16 bytes divides, in 32 bits
        {"name": "norm backward odd", "op": "norm_back", "rows": 1999, "n": 1030, "x": "f32", "w": "f32"},
        # serving: one sampled token with its 20 best alternatives
        {"name": "logprobs one token", "op": "logprobs", "rows": 1, "vocab": 131072, "x": "bf16", "top": 20, "masked": 0},
        # scoring the tokens of a batch
        {"name": "logprobs batch", "op": "logprobs", "rows": 4096, "vocab": 32000, "x": "bf16", "top": 0, "masked": 0},
        # a ragged batch in 32 bits, odd vocabulary, part of it masked out, with alternatives
        {"name": "logprobs odd top 5", "op": "logprobs", "rows": 300, "vocab": 50001, "x": "f32", "top": 5, "masked": 130},
        # the loss's gradient for a training batch
        {"name": "logprobs backward", "op": "logprobs_back", "rows": 8192, "vocab": 32000, "x": "bf16", "top": 0,
         "masked": 0},
        # with an entropy bonus and a term in the alternatives, ragged, in 32 bits
        {"name": "logprobs backward odd", "op": "logprobs_back", "rows": 129, "vocab": 37003, "x": "f32", "top": 8,
         "masked": 11},
        # the biases and norm weights that are not sketched
        {"name": "adamw biases", "op": "adamw", "total": 20000, "tensors": 25, "p": "f32", "g": "f32", "state": "f32",
         "copy": "none"},
        # a residual network's 62 tensors, views of one flat vector at whatever offset
        {"name": "adamw 62 tensors", "op": "adamw", "total": 11173962, "tensors": 62, "p": "f32", "g": "f32",
         "state": "f32", "copy": "none"},
        # a transformer's 90M parameters in 16 bits, the states in 8
        {"name": "adamw 8-bit states", "op": "adamw", "total": 90000000, "tensors": 150, "p": "bf16", "g": "bf16",
         "state": "e4m3", "copy": "none"},
    ]


def _log_uniform(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    n = n if rng.random() < 0.5 else max(lo, n // 64 * 64)     # odd sizes and round ones
    n = min(max(n, lo), hi)
    return n if n != 3072 else n + 8


def draw(rng):
    op = rng.choice(["norm", "norm_back", "logprobs", "logprobs_back", "adamw"])
    x = rng.choice(["f32", "bf16", "f16"])
    if op in ("norm", "norm_back"):
        n = _log_uniform(rng, 64, 16384)
        rows = _log_uniform(rng, 1, max(1, min(65536, (1 << 25) // n)))
        return {"op": op, "rows": rows, "n": n, "x": x, "w": rng.choice(["f32", x])}
    if op in ("logprobs", "logprobs_back"):
        vocab = _log_uniform(rng, 500, 200000)
        rows = _log_uniform(rng, 1, max(1, min(8192, (1 << 26) // vocab)))
        top = rng.choice([0, 0, 1, 5, 20])
        return {"op": op, "rows": rows, "vocab": vocab, "x": x, "top": top, "masked": rng.choice([0, vocab // 50])}
    state = rng.choice(["f32", "e4m3"])
    total = _log_uniform(rng, 5000, 30000000)
    p = rng.choice(["f32", "bf16"])
    return {"op": op, "total": total, "tensors": rng.randint(1, min(200, total // 64)), "p": p, "g": rng.choice([p, "f32"]),
            "state": state, "copy": rng.choice(["none", "bf16"]) if p == "f32" else "none"}


def work(case):
    if case["op"] in ("norm", "norm_back"):
        rows, n, ex = case["rows"], case["n"], BYTES[case["x"]]
        streams = 2 if case["op"] == "norm" else 3
        per_column = 2 * BYTES[case["w"]] if case["op"] == "norm" else BYTES[case["w"]] + 8
        return {"bytes": streams * rows * n * ex + per_column * n + 8 * rows, "flops": (8 if streams == 2 else 14) * rows * n}
    if case["op"] in ("logprobs", "logprobs_back"):
        rows, v, ex = case["rows"], case["vocab"], BYTES[case["x"]]
        streams = 1 if case["op"] == "logprobs" else 2
        return {"bytes": streams * rows * v * ex + rows * (20 + 8 * case["top"]), "flops": (6 if streams == 1 else 8) * rows * v}
    each = 2 * BYTES[case["p"]] + BYTES[case["g"]] + 4 * BYTES[case["state"]] + BYTES[case["copy"]]
    scales = 16 * (case["total"] // BLOCK) if case["state"] == "e4m3" else 0
    return {"bytes": each * case["total"] + scales, "flops": 15 * case["total"]}


def _library():
    global _ops
    if _ops is None:
        from paper_1903_04488_b200 import train_ops
        _ops = train_ops
    return _ops


# ---- inputs ------------------------------------------------------------------------------------------


def _sizes(total, tensors):
    """Lengths over a range of 1 : 1000, as a model's tensors have."""
    wts = [math.exp(math.log(1000.0) * ((i * 0.6180339887) % 1.0)) for i in range(tensors)]
    lens = [max(1, int(total * w / sum(wts))) for w in wts]
    lens[-1] += total - sum(lens)
    return lens


def _offsets(lens, pad):
    """Where each tensor starts in the flat vector; with `pad` at the next whole block."""
    ends = list(itertools.accumulate(-(-n // pad) * pad for n in lens))
    return [0] + ends[:-1], ends[-1]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    st = dict(case)
    dt = DTYPES.get(case.get("x"))
    if case["op"] in ("norm", "norm_back"):
        rows, n = case["rows"], case["n"]
        # activations: an offset per row, a few wide channels
        wide = 1 + 8 * (torch.rand(n, generator=gen, device="cuda") < 0.01)
        st["x"] = (rand(rows, n) * wide + 0.5 * rand(rows, 1) + 0.3).to(dt)
        st["w"] = (1 + 0.1 * rand(n)).to(DTYPES[case["w"]])
        st["b"] = (0.1 * rand(n)).to(DTYPES[case["w"]])
        if case["op"] == "norm_back":
            st["dy"] = (0.01 * rand(rows, n) + 0.002 * rand(n)).to(dt)
            x = st["x"].float()
            mean = x.mean(-1)
            st["stats"] = torch.stack([mean, ((x - mean[:, None]).square().mean(-1) + NORM_EPS).rsqrt()])
        return st
    if case["op"] in ("logprobs", "logprobs_back"):
        rows, v = case["rows"], case["vocab"]
        st["ids"] = torch.randint(0, v - case["masked"], (rows,), generator=gen, device="cuda")
        z = rand(rows, v).mul_(2.0)
        z.scatter_add_(1, st["ids"][:, None], 3 * rand(rows, 1) + 6)      # the model has learnt something
        if case["masked"]:
            z[:, v - case["masked"]:] = -math.inf                         # the padding of the vocabulary
        st["z"] = z.to(dt)
        del z
        if case["op"] == "logprobs_back":
            zf = st["z"].float()
            lse = zf.logsumexp(-1)
            logp = zf - lse[:, None]
            st["lse"], st["entropy"] = lse, -(logp.exp() * logp.clamp_min(-1e30)).sum(-1)
            st["d_logp"] = -torch.rand(rows, generator=gen, device="cuda") / rows
            st["d_entropy"] = 0.01 * rand(rows) / rows if case["top"] else None
            st["top_idx"] = st["d_top"] = None
            if case["top"]:
                # distinct alternatives of each row
                st["top_idx"] = zf.topk(case["top"], dim=1).indices.to(torch.int32)
                st["d_top"] = 0.1 * rand(rows, case["top"]) / rows
        return st
    lens = _sizes(case["total"], case["tensors"])
    small = case["state"] == "e4m3"
    starts, flat = _offsets(lens, BLOCK if small else 1)
    pdt, gdt = DTYPES[case["p"]], DTYPES[case["g"]]
    st["t"], st["seed"] = STEP0, seed
    mask = torch.zeros(flat, dtype=torch.bool, device="cuda")
    for s, n in zip(starts, lens):
        mask[s: s + n] = True
    # every 256 elements have gradients of one size, the states that go with it, and some zeros
    nb = -(-flat // BLOCK)
    size = torch.exp2(torch.randint(-16, -8, (nb, 1), generator=gen, device="cuda").float())
    spread = lambda t: (t.view(nb, -1) * size).view(-1)[:flat].mul_(mask)  # noqa: E731
    st["p"] = (0.02 * rand(flat) * mask).to(pdt)
    st["g"] = spread(rand(nb * BLOCK)).to(gdt)
    if small:
        codes = lambda t: (t.clamp(-448, 448) * mask).to(torch.float8_e4m3fn)  # noqa: E731
        st["m"], st["v"] = codes(100 * rand(flat)), codes(20 + 120 * rand(flat).abs())
        st["ms"], st["vs"] = size.view(-1) / 300, size.view(-1) / 100
        first = [s // BLOCK for s in starts] + [flat // BLOCK]
        st["first"] = torch.tensor(first, device="cuda")               # each tensor's first block
    else:
        st["m"], st["v"] = spread(0.3 * rand(nb * BLOCK)), spread(rand(nb * BLOCK)).square()
    st["copy_out"] = torch.zeros(flat, dtype=torch.bfloat16, device="cuda") if case["copy"] == "bf16" else None
    cut = lambda t: [t[s: s + n] for s, n in zip(starts, lens)]  # noqa: E731
    st["grads"] = cut(st["g"])
    if own:
        # the handle that a program keeps: which tensors, and where their states are
        scales = lambda t: [t[s // BLOCK: s // BLOCK + -(-n // BLOCK)] for s, n in zip(starts, lens)]  # noqa: E731
        st["opt"] = _library().AdamW(
            cut(st["p"]), lr=LR, betas=(BETA1, BETA2), eps=EPS, weight_decay=DECAY, state=case["state"],
            m=cut(st["m"]), v=cut(st["v"]), m_scale=scales(st["ms"]) if small else None,
            v_scale=scales(st["vs"]) if small else None, copies=cut(st["copy_out"]) if case["copy"] == "bf16" else None,
            step_count=STEP0)
    return st


# ---- one pass ----------------------------------------------------------------------------------------


def run(st):
    return (_run_own if own else _run_plain)(st)


def _run_own(st):
    train_ops = _ops or _library()
    op = st["op"]
    if op == "norm":
        y, stats = train_ops.layer_norm(st["x"], st["w"], st["b"], NORM_EPS)
        return {"y": y, "stats": stats}
    if op == "norm_back":
        dx, dw, db = train_ops.layer_norm_backward(st["dy"], st["x"], st["w"], st["stats"])
        return {"dx": dx, "dw": dw, "db": db}
    if op == "logprobs":
        r = train_ops.token_logprobs(st["z"], st["ids"], top=st["top"])
        return {"stats": r.stats, "top_idx": r.top_idx, "top_logp": r.top_logp}
    if op == "logprobs_back":
        return train_ops.token_logprobs_backward(st["z"], st["ids"], st["lse"], st["d_logp"], entropy=st["entropy"],
                                                 d_entropy=st["d_entropy"], top_idx=st["top_idx"], d_top=st["d_top"])
    st["t"] += 1
    st["opt"].step(st["grads"], seed=st["seed"] + st["t"] if st["state"] == "e4m3" else None)
    return _adamw_out(st)


def _adamw_out(st):
    names = ("p", "m", "v") + (("ms", "vs") if st["state"] == "e4m3" else ())
    return {k: st[k] for k in names + (("copy_out",) if st["copy_out"] is not None else ())}


def _run_plain(st):
    return {"norm": _norm, "norm_back": _norm_back, "logprobs": _logprobs, "logprobs_back": _logprobs_back,
            "adamw": _adamw}[st["op"]](st)


def _norm(st):
    x = st["x"].float()
    mean = x.mean(-1, keepdim=True)
    d = x - mean
    rstd = 1 / torch.sqrt((d * d).mean(-1, keepdim=True) + NORM_EPS)
    y = d * rstd * st["w"].float() + st["b"].float()
    return {"y": y.to(st["x"].dtype), "stats": torch.cat([mean, rstd], 1).t().contiguous()}


def _norm_back(st):
    x, dy = st["x"].float(), st["dy"].float()
    mean, rstd = st["stats"][0][:, None], st["stats"][1][:, None]
    h = (x - mean) * rstd
    a = dy * st["w"].float()
    dx = rstd * (a - a.mean(-1, keepdim=True) - h * (a * h).mean(-1, keepdim=True))
    return {"dx": dx.to(st["x"].dtype), "dw": (dy * h).sum(0), "db": dy.sum(0)}


def _top(z, k):
    """The k largest of each row, the lowest index first among equals: keys of value and index, none equal."""
    bits = (z + 0.0).view(torch.int32).to(torch.int64)
    order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
    v = z.shape[1]
    key = order * (1 << 32) + (v - 1 - torch.arange(v, device=z.device))
    best = key.topk(k, dim=1).values
    return (v - 1 - (best & 0xFFFFFFFF)).to(torch.int32)


def _logprobs(st):
    z = st["z"].float()
    m = z.amax(-1, keepdim=True)
    d = z - m
    e = torch.exp(d)
    s = e.sum(-1)
    log_s = torch.log(s)
    entropy = log_s - torch.where(e > 0, e * d, 0.0).sum(-1) / s
    logp = d.gather(1, st["ids"][:, None]).squeeze(1) - log_s
    out = {"stats": torch.stack([logp, entropy, m.squeeze(1) + log_s]), "top_idx": None, "top_logp": None}
    if st["top"]:
        out["top_idx"] = _top(z, st["top"])
        out["top_logp"] = d.gather(1, out["top_idx"].long()) - log_s[:, None]
    return out


def _logprobs_back(st):
    logp = st["z"].float() - st["lse"][:, None]
    p = torch.exp(logp)
    c = st["d_logp"]
    if st["top"]:
        c = c + st["d_top"].sum(-1)
    dz = -p * c[:, None]
    if st["d_entropy"] is not None:
        dz = dz - torch.where(p > 0, p * (logp + st["entropy"][:, None]), 0.0) * st["d_entropy"][:, None]
    dz.scatter_add_(1, st["ids"][:, None], st["d_logp"][:, None])
    if st["top"]:
        dz.scatter_add_(1, st["top_idx"].long(), st["d_top"])
    return dz.to(st["z"].dtype)


def _mix(x):
    """A mixing of 32 bits (in int64): the dither of a rounding comes from it."""
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _dither_word(st, nb):
    """32 bits for each element of each block, from the seed, the tensor's place in the list and the element's in it."""
    seed = torch.full((1,), (st["seed"] + st["t"]) & 0xFFFFFFFF, dtype=torch.int64, device="cuda")
    block = torch.arange(nb, device="cuda")
    tensor = torch.searchsorted(st["first"], block, right=True) - 1
    key = _mix((_mix(_mix(seed)) + tensor) & 0xFFFFFFFF)                  # the seed's upper half is zero here
    at = (block - st["first"][tensor])[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")
    return _mix(key[:, None] ^ at)


def _to_e4m3(x, u):
    """Codes and scales of blocks x [nb, 256] of magnitudes: value / scale, rounded down after adding u in [0, 1) steps."""
    amax = x.amax(-1, keepdim=True)
    tiny = amax < 2.0 ** -100
    y = (x * torch.where(tiny, 0.0, 448.0 / amax)).clamp_max(448.0)
    e = ((y.view(torch.int32) >> 23) - 121).clamp_min(0)
    n = torch.floor(y * ((136 - e) << 23).view(torch.float32) + u).to(torch.int32)
    return (e * 8 + n).clamp_max(126), torch.where(tiny, 0.0, amax / 448.0).squeeze(1)


def _adamw(st):
    st["t"] += 1
    t, small = st["t"], st["state"] == "e4m3"
    p, g = st["p"].float(), st["g"].float()
    if small:
        p, g = p.view(-1, BLOCK), g.view(-1, BLOCK)
        m = st["m"].float().view(-1, BLOCK) * st["ms"][:, None]
        v = (st["v"].float().view(-1, BLOCK) * st["vs"][:, None]).square()
    else:
        m, v = st["m"], st["v"]
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g * g * (1 - BETA2)
    r = torch.sqrt(v)
    p = p * (1 - LR * DECAY) - (LR / (1 - BETA1 ** t)) * (m / (r / math.sqrt(1 - BETA2 ** t) + EPS))
    if small:
        word = _dither_word(st, p.shape[0])
        half = 2.0 ** -17
        code, st_ms = _to_e4m3(m.abs(), (word & 0xFFFF).float() * 2.0 ** -16 + half)
        code = code + (m < 0) * 128
        st["m"].copy_(code.to(torch.uint8).view(torch.float8_e4m3fn).view(-1))
        st["ms"].copy_(st_ms)
        code, st_vs = _to_e4m3(r, (word >> 16).float() * 2.0 ** -16 + half)
        code = torch.where(r > 0, code.clamp_min(1), code)
        st["v"].copy_(code.to(torch.uint8).view(torch.float8_e4m3fn).view(-1))
        st["vs"].copy_(st_vs)
        if st["p"].dtype == torch.bfloat16:
            bits = p.view(torch.int32).to(torch.int64) + ((word * 0x9E3779B9 & 0xFFFFFFFF) >> 16)
            p = (bits & ~0xFFFF).to(torch.int32).view(torch.float32)
    else:
        st["m"].copy_(m)
        st["v"].copy_(v)
    st["p"].copy_(p.view(-1))
    if st["copy_out"] is not None:
        st["copy_out"].copy_(p.view(-1))
    return _adamw_out(st)


# ---- the definitions in 64 bits ----------------------------------------------------------------------


def exact(case, seed):
    global own
    mine, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = mine
    f = lambda k: st[k].to(torch.float64)  # noqa: E731
    if case["op"] == "norm":
        x = f("x")
        var, mean = torch.var_mean(x, -1, correction=0)
        rstd = (var + NORM_EPS) ** -0.5
        y = torch.addcmul(f("b"), (x - mean[:, None]) * rstd[:, None], f("w"))
        return {"y": y, "stats": torch.stack([mean, rstd])}
    if case["op"] == "norm_back":
        # y = w h + b with h = (x - mean) rstd, and dh/dx = rstd (I - 1 1'/n - h h'/n)
        n = case["n"]
        h = torch.addcmul(-(f("stats")[0] * f("stats")[1])[:, None], f("x"), f("stats")[1][:, None])
        dh = f("dy") * f("w")
        along = torch.einsum("rn,rn->r", dh, h) / n
        dx = (dh - dh.sum(1, keepdim=True) / n - along[:, None] * h) * f("stats")[1][:, None]
        return {"dx": dx, "dw": torch.einsum("rn,rn->n", f("dy"), h), "db": f("dy").sum(0)}
    if case["op"] == "logprobs":
        logp = torch.log_softmax(f("z"), -1)
        h = -(logp.exp() * logp.nan_to_num(neginf=0.0)).sum(-1)
        out = {"stats": torch.stack([logp[torch.arange(case["rows"], device="cuda"), st["ids"]], h,
                                     torch.logsumexp(f("z"), -1)]), "top_idx": None, "top_logp": None}
        if case["top"]:
            out["top_logp"] = logp.topk(case["top"], dim=1).values
        return out
    if case["op"] == "logprobs_back":
        # the statistics are inputs: p = exp(z - lse)
        logp = f("z") - f("lse")[:, None]
        p = logp.exp()
        dz = torch.zeros_like(p)
        rows = torch.arange(case["rows"], device="cuda")
        dz[rows, st["ids"]] += f("d_logp")
        weight = f("d_logp")
        if case["top"]:
            dz.scatter_add_(1, st["top_idx"].long(), f("d_top"))
            weight = weight + f("d_top").sum(1)
            dz -= p * (logp.nan_to_num(neginf=0.0) + f("entropy")[:, None]) * f("d_entropy")[:, None]
        return dz - p * weight[:, None]
    small, t = case["state"] == "e4m3", STEP0 + 1
    spread = lambda s: s.double().repeat_interleave(BLOCK)  # noqa: E731
    m0 = f("m") * spread(st["ms"]) if small else f("m")
    v0 = (f("v") * spread(st["vs"])) ** 2 if small else f("v")
    m1 = BETA1 * m0 + (1 - BETA1) * f("g")
    v1 = BETA2 * v0 + (1 - BETA2) * f("g") ** 2
    upd = (m1 / (1 - BETA1 ** t)) / ((v1 / (1 - BETA2 ** t)).sqrt() + EPS)
    p1 = f("p") - LR * (DECAY * f("p") + upd)
    out = {"p": p1, "m": m1, "v": v1}
    if small:
        # the codes before their rounding: an eighth of a code is lost by it on either side
        blocks = lambda q: q.abs().view(-1, BLOCK).amax(1) / 448  # noqa: E731
        out["ms"], out["vs"] = blocks(m1), blocks(v1.sqrt())
        code = lambda q, s: torch.where(s > 0, q.view(-1, BLOCK).T / s, 0.0).T.reshape(-1)  # noqa: E731
        out["m"], out["v"] = code(m1, out["ms"]), code(v1.sqrt(), out["vs"])
    if st["copy_out"] is not None:
        out["copy_out"] = p1
    return out
