"""Log probabilities where logits are large: masks of -1e9 to -1e20, in front, behind, at random and everywhere, and rows far from zero.

Tolerances (u = 2^-24): a sum of a chain of c additions is within c u; the constants and roundings between a logit and its log
probability are six, each relative to the result (log2 e, its product with the scale, the multiplication, two sums, log 2)."""
import math

import numpy as np
import pytest
import torch

from paper_1903_04488_b200 import train_ops as T

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


def definition(z, ids, scale):
    z = z.double() * float(np.float32(scale))
    m = z.amax(-1, keepdim=True)
    log_s = (z - m).exp().sum(-1, keepdim=True).log()
    logp = (z - m) - log_s
    p = logp.exp()
    h = -torch.where(p > 0, p * logp, 0.0).sum(-1)
    return logp.gather(1, ids[:, None]).squeeze(1), h, (m + log_s).squeeze(1), logp, p


def rows_of(kind, value, rows, v, dtype, gen):
    z = 2 * torch.randn(rows, v, generator=gen, device="cuda")
    if kind == "all":
        z[:] = value
    elif kind == "front":
        z[:, : v // 2] = value
    elif kind == "behind":
        z[:, v // 2:] = value
    elif kind == "random":
        z = torch.where(torch.rand(rows, v, generator=gen, device="cuda") < 0.7, value, z)
    elif kind == "one left":
        z[:] = value
        z[:, v // 3] = 1.5
    elif kind == "far":                        # neighbouring numbers of 32 bits, far above zero
        step = 2.0 ** (math.floor(math.log2(-value)) - 23)
        z = -value + step * torch.randint(0, 12, (rows, v), generator=gen, device="cuda").float()
    return z.to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("value", [-1e6, -1e8, -1e9, -1e10, -1e12, -1e15, -1e20, -1e28])
@pytest.mark.parametrize("kind", ["all", "front", "behind", "random", "one left", "far"])
def test_logprobs_of_large_logits(cuda_device, kind, value, dtype):
    gen = torch.Generator(device="cuda").manual_seed(7)
    for rows, v in ((3, 40001), (1, 131072), (700, 3001)):
        z = rows_of(kind, value, rows, v, dtype, gen)
        ids = torch.randint(0, v, (rows,), generator=gen, device="cuda")
        ids[0] = z[0].argmax()
        for scale in (0.1, 1.0, 10.0):
            logp, h, lse, every, p = definition(z, ids, scale)
            rel = (v / 256 + 64) * U + 4 * U * (h + 4)
            for top in (0, 7):
                r = T.token_logprobs(z, ids, top=top, scale=scale)
                for name, got, want, tol in (("logp", r.logp, logp, rel + 6 * U * logp.abs()), ("entropy", r.entropy, h, (rel + 4 * U) * (h + 4)),
                                             ("lse", r.lse, lse, rel + 6 * U * lse.abs())):
                    err = (got.double() - want).abs()
                    assert (err <= tol).all(), f"{name}, {rows} x {v}, scale {scale}, top {top}: got {got.tolist()[:3]}, should be {want.tolist()[:3]}"
                if top:
                    order = z.float().sort(dim=1, descending=True, stable=True).indices[:, :top]
                    assert torch.equal(r.top_idx.long(), order)
                    want = every.gather(1, order)
                    assert ((r.top_logp.double() - want).abs() <= rel[:, None] + 6 * U * want.abs()).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("value", [-1e9, -1e10, -1e12, -1e20])
@pytest.mark.parametrize("kind", ["all", "front", "behind", "random", "one left", "far"])
def test_gradient_of_large_logits(cuda_device, kind, value, dtype):
    gen = torch.Generator(device="cuda").manual_seed(8)
    rows, v = 5, 9001
    z = rows_of(kind, value, rows, v, dtype, gen)
    ids = torch.randint(0, v, (rows,), generator=gen, device="cuda")
    d, dh = (torch.randn(rows, generator=gen, device="cuda") for _ in range(2))
    d[1] = dh[1] = 0.0                         # a row that the loss leaves out
    for scale in (0.1, 1.0, 10.0, 0.37):
        r = T.token_logprobs(z, ids, scale=scale)
        for kw in ({}, dict(entropy=r.entropy, d_entropy=dh)):
            out = T.token_logprobs_backward(z, ids, r.lse, d, scale=scale, **kw)
            assert out.isfinite().all() and not out[1].any()
            # a probability is at most 1, and p |log p| at most 1 / e, whatever lse has lost to its 32 bits
            most = scale * (2 * d.abs() + (dh.abs() * (1 + r.entropy) if kw else 0)) * (1 + 2 * HALF[dtype]) + 1e-30
            assert (out.float().abs() <= most[:, None]).all()
            if kind in ("all", "far"):
                continue                       # lse itself does not tell such logits apart
            _, h, lse, logp, p = definition(z, ids, scale)
            one = torch.zeros_like(p).scatter_(1, ids[:, None], d.double()[:, None])
            gh = dh.double()[:, None] if kw else 0.0
            lp = torch.where(p > 0, logp, 0.0)
            want = scale * (one - p * (d.double()[:, None] + gh * (lp + h[:, None])))
            # lse and entropy come with the forward pass's tolerance
            given = (v / 256 + 64) * U + 4 * U * (h + 4) + 6 * U * lse.abs()
            relp = (8 * U + 6 * U * lp.abs()) + given[:, None]
            size = d.double().abs()[:, None] + (gh * 1.0).abs() * (lp.abs() + h[:, None]) if kw else d.double().abs()[:, None]
            # 2^x below the smallest normal number is 0
            tol = scale * ((p * (relp + 40 * U) + 2.0 ** -126) * size + 40 * U * one.abs() + (p * (gh * 1.0).abs() * 2 * (given * (1 + h) + 4 * U * (h + 4))[:, None] if kw else 0.0))
            near = (out.double() - want).abs() <= tol + HALF[dtype] * (want.abs() + tol) + 1e-37
            assert near.all(), f"scale {scale}: {int((~near).sum())} outside"
