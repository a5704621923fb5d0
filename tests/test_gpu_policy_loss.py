"""The clipped policy loss and its gradient against the formula in 64 bits.

Tolerances are forward error bounds with U = 2^-24.  A row's log sum exp is a chain of roundings of which the longest is what a
thread adds up, v / 256 + 64 with the joins; 2^x is good to 2 units of its argument's weight (as for the log probabilities).  What
follows from it is bounded to first order: an error d of logp changes the ratio by ratio d, the divergence by (e^q - 1) d, its slope by
e^q d.  Gradients in 16 bits may take log2 p with one rounding more, of at most 2^-18."""
import math

import numpy as np
import pytest
import torch

from paper_1903_04488_b200 import autograd as A
from paper_1903_04488_b200 import train_ops as T

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def strided(x, pad, offset):
    rows, n = x.shape
    buf = torch.full((offset + rows * (n + pad),), 7.0, dtype=x.dtype, device=x.device)
    v = buf[offset: offset + rows * (n + pad)].view(rows, n + pad)[:, :n]
    v.copy_(x)
    return v


def near(got, want, tol, what):
    assert torch.equal(got.isnan(), want.isnan()), what
    same = ~want.isfinite()
    assert torch.equal(got.double()[same].nan_to_num(7.0, 8.0, 9.0), want[same].nan_to_num(7.0, 8.0, 9.0)), what
    err = torch.where(same, 0.0, (got.double() - want).abs())
    bad = err > torch.where(same, 0.0, tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} outside, worst {float((err / tol.clamp_min(1e-300))[bad].max()):.3g} of the bound"


def inputs(rows, v, dtype, seed, low, high, ref=True, weights=True, scale=1.0):
    g = gen(seed)
    z = (2 * torch.randn(rows, v, generator=g, device="cuda")).to(dtype)
    ids = torch.randint(0, v, (rows,), generator=g, device="cuda")
    logp = torch.log_softmax(z.double() * scale, -1).gather(1, ids[:, None]).squeeze(1)
    moved = 0.3 * torch.randn(rows, generator=g, device="cuda", dtype=torch.float64)
    for border in (1 - low, 1 + high):
        if 0 < border < math.inf:
            moved = torch.where((moved - math.log(border)).abs() < 1e-2, moved + 3e-2, moved)
    args = dict(old_logp=(logp - moved).float(), advantages=torch.randn(rows, generator=g, device="cuda"))
    args["ref_logp"] = (logp + 0.5 * torch.randn(rows, generator=g, device="cuda")).float() if ref else None
    w = torch.rand(rows, generator=g, device="cuda") / rows
    args["weights"] = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.2, 0.0, w) if weights else None
    return z, ids, args


def formula(z, ids, old_logp, advantages, ref_logp, weights, clip, kl, entropy, scale):
    """(stats, their tolerances, gradient, its tolerance) in 64 bits"""
    rows, v = z.shape
    scale, kl, entropy, low, high = (float(np.float32(x)) for x in (scale, kl, entropy, *clip))
    zs = z.double() * scale
    m = zs.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    log_s = (zs - m).exp().sum(-1, keepdim=True).log()
    lp = torch.where(zs == -math.inf, -math.inf, (zs - m) - log_s)
    p = lp.exp()
    flat = torch.where(p > 0, lp, 0.0)
    h = -(p * flat).sum(-1)
    inside = (ids >= 0) & (ids < v)
    at = ids.clamp(0, v - 1).long()[:, None]
    logp = lp.gather(1, at).squeeze(1)
    w = torch.ones(rows, dtype=torch.float64, device="cuda") if weights is None else weights.double()
    live = inside & (w != 0)
    adv, old = advantages.double(), old_logp.double()
    d_lp = (v / 256 + 64) * U + 4 * U * (h + 4) + 4 * U * torch.where(logp.isfinite(), logp.abs(), 0.0)
    ratio = (logp - old).exp()
    d_ratio = ratio * (1.01 * (d_lp + 2 * U * ((logp - old).abs() + old.abs()).nan_to_num(posinf=0.0)) + 4 * U)
    kept = torch.where(adv >= 0, ratio.clamp_max(1 + high), ratio.clamp_min(1 - low))
    loss = -kept * adv - entropy * h
    along = torch.where(kept == ratio, -adv * ratio, 0.0)
    d_h = (d_lp + 8 * U) * (h + 4)
    d_loss = adv.abs() * (d_ratio + 4 * U * kept.nan_to_num(posinf=0.0)) + abs(entropy) * (d_h + 4 * U * h)
    d_along = adv.abs() * (d_ratio + 4 * U * ratio)
    big = torch.zeros_like(logp)
    k = torch.zeros_like(logp)
    d_k = torch.zeros_like(logp)
    if ref_logp is not None:
        q = ref_logp.double() - logp
        k = torch.expm1(q) - q
        d_q = d_lp + 2 * U * (q.abs() + ref_logp.double().abs())
        d_k = torch.expm1(q).abs() * d_q + q.exp() * d_q ** 2 + 4 * U * (torch.expm1(q).abs() + q.abs())
        loss, along = loss + kl * k, along - kl * torch.expm1(q)
        d_loss = d_loss + kl * (d_k + 4 * U * k)
        d_along = d_along + kl * (q.exp() * d_q + 8 * U * torch.expm1(q).abs())
        big = kl * k
    stats = torch.where(live, torch.stack([w * loss, logp, h, k, ratio]), 0.0)
    d_stats = torch.stack([w.abs() * (d_loss + 8 * U * (kept.nan_to_num(posinf=0.0) * adv.abs() + big + abs(entropy) * h)), d_lp, d_h, d_k, d_ratio])
    one = torch.zeros_like(p).scatter_(1, at, 1.0)
    ws = (w * scale)[:, None]
    grad = ws * (along[:, None] * (one - p) + entropy * p * (flat + h[:, None]))
    rel_p = d_lp[:, None] + 8 * U + 8 * U * flat.abs() + (2.0 ** -18 if z.dtype != torch.float32 else 0.0)
    size = along.abs()[:, None] + abs(entropy) * (flat.abs() + h[:, None])
    tol = ws.abs() * ((one + p) * d_along[:, None] + p * (rel_p + 16 * U) * size + abs(entropy) * p * (rel_p + d_h[:, None]) + 16 * U * one * along.abs()[:, None])
    grad = torch.where(live[:, None], grad, 0.0)
    return stats, d_stats, grad, tol


def check(z, ids, args, r, clip=(0.2, 0.2), kl=0.0, entropy=0.0, scale=1.0):
    stats, d_stats, grad, tol = formula(z, ids, **args, clip=clip, kl=kl, entropy=entropy, scale=scale)
    for i, name in enumerate(("loss", "logp", "entropy", "kl", "ratio")):
        near(r.stats[i], stats[i], d_stats[i] + 1e-37, name)
    if r.dlogits is not None:
        near(r.dlogits, grad, tol + HALF[z.dtype] * (grad.abs() + tol) + TINY[z.dtype] + 1e-37, "dlogits")


SIZES = [(1, 1), (3, 5), (2, 33), (7, 300), (65, 1000), (4, 2049), (3, 8200), (2, 40001), (1, 131072), (700, 517), (640, 8000), (5, 70001)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,v", SIZES)
def test_policy_loss(cuda_device, rows, v, dtype):
    for clip, kl, entropy, scale in (((0.2, 0.28), 0.0, 0.0, 1.0), ((0.1, 0.1), 0.3, 0.02, 0.7), ((1.0, math.inf), 0.0, -0.05, 1.0)):
        kw = dict(clip=clip, kl=kl, entropy=entropy, scale=scale)
        z, ids, args = inputs(rows, v, dtype, rows + v, *clip, ref=kl > 0, weights=kl > 0, scale=scale)
        r = T.policy_loss(z, ids, **args, **kw)
        check(z, ids, args, r, **kw)
        again = T.policy_loss(z, ids.to(torch.int32), **args, **kw)
        assert torch.equal(r.stats, again.stats) and torch.equal(r.dlogits, again.dlogits)
        bare = T.policy_loss(z, ids, **args, need_grad=False, **kw)
        assert bare.dlogits is None and torch.allclose(bare.stats, r.stats, rtol=1e-5, atol=1e-5)
        over = z.clone()
        assert torch.equal(T.policy_loss(over, ids, **args, out=over, **kw).dlogits, r.dlogits) and torch.equal(over, r.dlogits)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("v,pad,offset", [(1000, 24, 8), (1001, 2, 1), (999, 9, 3), (30011, 1, 5), (6, 3, 1)])
def test_policy_loss_of_strided_rows(cuda_device, dtype, v, pad, offset):
    z, ids, args = inputs(5, v, dtype, v, 0.2, 0.2)
    a = T.policy_loss(z, ids, **args, kl=0.1, entropy=0.01)
    check(z, ids, args, a, kl=0.1, entropy=0.01)
    zs = strided(z, pad, offset)
    for out in (None, strided(z, pad, offset), strided(z, pad + 1, offset + 1)):
        b = T.policy_loss(zs, ids, **args, kl=0.1, entropy=0.01, out=out)
        check(z, ids, args, b, kl=0.1, entropy=0.01)
        if out is not None:
            assert (out._base[:offset] == 7).all()
            assert (out.as_strided((4, out.stride(0) - v), out.stride(), out.storage_offset() + v) == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("v", [2500, 40000])
def test_policy_loss_masks(cuda_device, dtype, v):
    """-inf and the type's lowest value as masks, one logit left, far logits; rows that are not read hold anything."""
    low = torch.finfo(dtype).min
    z, ids, args = inputs(10, v, dtype, 4, 0.2, 0.2)
    args["weights"] = torch.rand(10, device="cuda", generator=gen(1)) + 0.1
    z[0, 100:] = -math.inf
    z[1] = math.nan                           # weight 0
    z[2] = low                                # everything masked with the lowest value: uniform
    z[3, 1:] = low
    z[4] = -math.inf
    z[4, 1777] = 3.0                          # one left
    z[5, ::2] = -math.inf
    z[6, :2049] = -math.inf                   # whole threads see nothing at first
    z[7] = math.inf                           # an id outside the vocabulary
    z[8] = torch.where(torch.rand(v, generator=gen(1), device="cuda") < 0.5, low, z[8])
    z[9] += 3000.0 if dtype != torch.float16 else 900.0
    ids = torch.tensor([5, 3, 7, 0, 1777, 1, 2300, v, -100, v - 1], device="cuda")
    args["weights"][1] = 0
    lp = torch.log_softmax(z.double(), -1).gather(1, ids.clamp(0, v - 1)[:, None]).squeeze(1).nan_to_num(0.0)
    args["old_logp"], args["ref_logp"] = (lp - 0.05).float(), (lp + 0.1).float()
    r = T.policy_loss(z, ids, **args, kl=0.1, entropy=0.01)
    check(z, ids, args, r, kl=0.1, entropy=0.01)
    for i in (1, 7, 8):
        assert (r.stats[:, i] == 0).all() and (r.dlogits[i] == 0).all()


def test_policy_loss_of_masked_tokens_empty_rows_and_values_that_are_not_finite(cuda_device):
    z, ids, args = inputs(6, 3001, torch.float32, 8, 0.2, 0.2, ref=False, weights=False)
    args["advantages"] = torch.tensor([1.0, -1.0, 1.0, 0.0, 1.0, 1.0], device="cuda")
    z[0, ids[0]] = z[1, ids[1]] = -math.inf   # a token that cannot be drawn any more: ratio 0, not clipped below for A > 0
    z[2] = -math.inf                          # nothing left
    args["old_logp"][3] = -500.0              # the ratio overflows, the advantage is 0
    z[4, 77] = math.nan
    z[5, 78] = math.inf
    r = T.policy_loss(z, ids, **args, entropy=0.01)
    assert r.logp[0] == -math.inf and r.ratio[0] == 0 and r.dlogits[0].isfinite().all() and r.dlogits[0, ids[0]] == 0
    assert r.ratio[1] == 0 and abs(float(r.loss[1]) - 0.8 + 0.01 * float(r.entropy[1])) < 1e-5
    assert r.logp[2] == -math.inf and r.entropy[2] == 0 and (r.dlogits[2] == 0).all()
    assert r.ratio[3] == math.inf and r.loss[3].isfinite() and r.dlogits[3].isfinite().all()
    assert r.stats[:3, 4:].isnan().all() and r.dlogits[4:].isnan().any(1).all()


def test_policy_loss_of_rows_that_do_not_fit_shared_memory(cuda_device):
    v = 900001
    z, ids, args = inputs(2, v, torch.bfloat16, 5, 0.2, 0.2)
    check(z, ids, args, T.policy_loss(z, ids, **args, kl=0.1, entropy=0.01), kl=0.1, entropy=0.01)
    z, ids, args = inputs(1, v, torch.float32, 6, 0.2, 0.2)
    r = T.policy_loss(z, ids, **args, kl=0.1)
    check(z, ids, args, r, kl=0.1)
    over = z.clone()
    assert torch.equal(T.policy_loss(over, ids, **args, kl=0.1, out=over).dlogits, r.dlogits)


def test_policy_loss_of_no_rows_and_long_offsets(cuda_device):
    e = lambda *s, **k: torch.empty(*s, device="cuda", **k)  # noqa: E731
    r = T.policy_loss(e(0, 9), e(0, dtype=torch.int64), e(0), e(0))
    assert r.stats.shape == (5, 0) and r.dlogits.shape == (0, 9)
    v, rows = 1 << 20, 4200                    # 4.4e9 logits: rows beyond 2^32 elements
    z = torch.zeros(rows, v, dtype=torch.bfloat16, device="cuda")
    ids = torch.full((rows,), 3, device="cuda")
    w = torch.zeros(rows, device="cuda")
    w[0] = w[-1] = 1
    z[0, :7] = z[-1, :7] = torch.arange(7, device="cuda").to(torch.bfloat16)
    old, adv = torch.full((rows,), -13.0, device="cuda"), torch.ones(rows, device="cuda")
    r = T.policy_loss(z, ids, old, adv, weights=w, out=z)
    assert torch.equal(r.stats[:, 0], r.stats[:, -1]) and r.ratio[0] > 1.2
    assert (z[0] == 0).all() and (z[-1] == 0).all()            # clipped: no gradient
    assert (r.stats[:, 1:-1] == 0).all() and (z[rows // 2] == 0).all()
    z[0, :7] = z[-1, :7] = torch.arange(7, device="cuda").to(torch.bfloat16)
    r = T.policy_loss(z, ids, old, -adv, weights=w, out=z)     # not clipped where the advantage is negative
    assert torch.equal(r.stats[:, 0], r.stats[:, -1]) and torch.equal(z[0], z[-1]) and z[0, 3] > 0


def test_policy_loss_gradient_against_differences(cuda_device):
    z, ids, args = inputs(6, 41, torch.float32, 9, 0.2, 0.28)
    kw = dict(clip=(0.2, 0.28), kl=0.2, entropy=0.03, scale=1.3)
    zr = z.clone().requires_grad_()
    up = torch.rand(6, device="cuda", generator=gen(3))
    (A.policy_loss(zr, ids, args["old_logp"], args["advantages"], ref_logp=args["ref_logp"], weights=args["weights"], **kw)[0] * up).sum().backward()
    f = lambda z: float((formula(z, ids, **args, **kw)[0][0] * up).sum())  # noqa: E731
    for seed in range(4):
        d = torch.randn(z.shape, generator=gen(seed), device="cuda", dtype=torch.float64)
        step = 1e-5
        want = (f(z.double() + step * d) - f(z.double() - step * d)) / (2 * step)
        got = (zr.grad.double() * d).sum()
        size = float((zr.grad.double() * d).abs().sum())
        # 64-bit differences: step^2 and cancellation over 2 step; the gradient: some 100 units
        assert abs(float(got) - want) <= 200 * U * size + 1e-7 * size + 1e-9


def test_policy_loss_on_another_stream_in_graphs_and_through_autograd(cuda_device):
    z, ids, args = inputs(300, 5000, torch.bfloat16, 2, 0.2, 0.2)
    want = T.policy_loss(z, ids, **args, kl=0.1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = T.policy_loss(z, ids, **args, kl=0.1)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got.stats, want.stats) and torch.equal(got.dlogits, want.dlogits)
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(T.policy_loss(z, ids, **args, kl=0.1))
        graphs.append(g)
    z.mul_(0.5)
    want = T.policy_loss(z, ids, **args, kl=0.1)
    for g, got in zip(graphs, outs):
        g.replay()
        assert torch.equal(got.stats, want.stats) and torch.equal(got.dlogits, want.dlogits)
    # through autograd: not in rows, and with the same gradient twice
    zr = z.t().contiguous().t().requires_grad_()
    loss, logp, entropy, kl, ratio = A.policy_loss(zr, ids, args["old_logp"], args["advantages"], ref_logp=args["ref_logp"], weights=args["weights"], kl=0.1)
    assert not logp.requires_grad and not ratio.requires_grad
    loss.sum().backward(retain_graph=True)
    first = zr.grad.clone()
    assert torch.equal(first, want.dlogits)
    loss.sum().backward()
    assert torch.equal(zr.grad, first + first)
    assert torch.allclose(torch.stack([loss, logp, entropy, kl, ratio]), want.stats, rtol=1e-4, atol=1e-6)
