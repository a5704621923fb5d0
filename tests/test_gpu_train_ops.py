"""Layer norm, log probabilities of given tokens and AdamW against plain forms in 64 bits.

Tolerances are forward error bounds with u = 2^-24: a sum of a chain of c additions of terms t_i is within c u sum |t_i|, one
rounding to a 16-bit format adds half a unit of its last place.  `CHAIN` covers the longest chain of a row sum (64
elements per thread, 10 levels of a tree) with the roundings around it."""
import math

import numpy as np
import pytest
import torch

from paper_1903_04488_b200 import autograd as A
from paper_1903_04488_b200 import ssgd as S
from paper_1903_04488_b200 import train_ops as T

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
CHAIN = 200
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # 24, 8 and 11 significant bits
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}   # half the last place of a subnormal
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def near(got, want, tol, what=""):
    err = (got.double() - want).abs()
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} outside, worst {float((err / tol.clamp_min(1e-300))[bad].max()):.3g} of the bound"


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def strided(x, pad, offset):
    """The same values as a view with `pad` elements between rows, `offset` elements into its buffer."""
    rows, n = x.shape
    buf = torch.full((offset + rows * (n + pad),), 7.0, dtype=x.dtype, device=x.device)
    v = buf[offset: offset + rows * (n + pad)].view(rows, n + pad)[:, :n]
    v.copy_(x)
    return v


# ---- layer norm --------------------------------------------------------------------------------------

NORM_SIZES = [(1, 1), (3, 7), (5, 64), (33, 512), (9, 513), (17, 1030), (70, 2048), (4, 4096), (3, 4100), (5, 8192), (2, 16384),
              (3, 16390), (2, 20001), (300, 96), (1, 65536), (2500, 40)]


def norm_inputs(rows, n, dtype, seed, wdtype=None):
    g = gen(seed)
    x = (torch.randn(rows, n, generator=g, device="cuda") * 2 + torch.randn(rows, 1, generator=g, device="cuda")).to(dtype)
    w = (1 + 0.3 * torch.randn(n, generator=g, device="cuda")).to(wdtype or torch.float32)
    b = torch.randn(n, generator=g, device="cuda").to(wdtype or torch.float32)
    dy = torch.randn(rows, n, generator=g, device="cuda").to(dtype)
    return x, w, b, dy


def norm64(x, w, b, eps):
    x = x.double()
    mean = x.mean(-1, keepdim=True)
    rstd = ((x - mean).square().mean(-1, keepdim=True) + eps).rsqrt()
    h = (x - mean) * rstd
    return (h * w.double() if w is not None else h) + (b.double() if b is not None else 0), mean, rstd, h


def check_norm(x, w, b, eps, y, stats):
    want, mean, rstd, h = norm64(x, w, b, eps)
    size = x.double().abs().mean(-1, keepdim=True)
    near(stats[0][:, None], mean, CHAIN * U * size + 1e-300, "mean")
    # the variance's error: its chain, and the mean's own error, which enters squared
    rel = CHAIN * U + (CHAIN * U * size * rstd) ** 2
    near(stats[1][:, None], rstd, rel * rstd, "rstd")
    wa = w.double().abs() if w is not None else 1.0
    ba = b.double().abs() if b is not None else 0.0
    tol = (CHAIN * U * rstd * size + rel * h.abs()) * wa + 4 * U * ba
    near(y, want, tol + HALF[x.dtype] * (want.abs() + tol) + TINY[x.dtype], "y")


def check_norm_back(x, w, stats, dy, dx, dw, db):
    x, d = x.double(), dy.double()
    mean, rstd = stats[0].double()[:, None], stats[1].double()[:, None]
    h = (x - mean) * rstd
    a = d * w.double() if w is not None else d
    c1, c2 = a.mean(-1, keepdim=True), (a * h).mean(-1, keepdim=True)
    want = rstd * (a - c1 - h * c2)
    s1, s2 = a.abs().mean(-1, keepdim=True), (a * h).abs().mean(-1, keepdim=True)
    tol = CHAIN * U * rstd * (a.abs() + s1 + h.abs() * s2)
    near(dx, want, tol + HALF[dy.dtype] * (want.abs() + tol) + TINY[dy.dtype], "dx")
    if dw is not None:
        near(dw, (d * h).sum(0), CHAIN * U * (d * h).abs().sum(0) + 1e-300, "dw")
        near(db, d.sum(0), CHAIN * U * d.abs().sum(0) + 1e-300, "db")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n", NORM_SIZES)
def test_norm_and_its_gradient(cuda_device, rows, n, dtype):
    x, w, b, dy = norm_inputs(rows, n, dtype, rows * 31 + n, dtype if (rows + n) % 2 else torch.float32)
    eps = 1e-5
    y, stats = T.layer_norm(x, w, b, eps)
    check_norm(x, w, b, eps, y, stats)
    dx, dw, db = T.layer_norm_backward(dy, x, w, stats)
    assert dw.dtype == db.dtype == torch.float32 and dx.dtype == dtype
    check_norm_back(x, w, stats, dy, dx, dw, db)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n", [(1500, 1000), (1301, 2048), (1202, 4096), (1187, 8192), (1300, 130), (2401, 512), (1250, 77), (701, 8704),
                                    (403, 12000)])
def test_norm_of_many_rows(cuda_device, rows, n, dtype):
    """More rows than the blocks take in their first turns, and a last turn that is not full."""
    x, w, b, dy = norm_inputs(rows, n, dtype, rows + n, torch.float32 if n % 3 else dtype)
    y, stats = T.layer_norm(x, w, b, 1e-5)
    check_norm(x, w, b, 1e-5, y, stats)
    dx, dw, db = T.layer_norm_backward(dy, x, w, stats)
    check_norm_back(x, w, stats, dy, dx, dw, db)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,pad,offset", [(512, 8, 8), (512, 1, 3), (2048, 2, 2), (1000, 24, 5), (20000, 7, 1)])
def test_norm_of_strided_rows(cuda_device, dtype, n, pad, offset):
    x, w, b, dy = norm_inputs(21, n, dtype, n + pad)
    xs, dys = strided(x, pad, offset), strided(dy, pad + 1, offset + 1)
    out, dxo = strided(x, pad + 3, offset), strided(x, pad, offset)
    y, stats = T.layer_norm(xs, w, b, 1e-5, out=out)
    check_norm(x, w, b, 1e-5, y, stats)
    assert (out._base[:offset] == 7).all() and (out.as_strided((21, pad + 3), out.stride(), out.storage_offset() + n)[:-1] == 7).all()
    dx, dw, db = T.layer_norm_backward(dys, xs, w, stats, dx=dxo)
    check_norm_back(x, w, stats, dy, dx, dw, db)
    assert (dxo._base[:offset] == 7).all()


def test_norm_without_parameters_in_place_and_accumulating(cuda_device):
    x, w, b, dy = norm_inputs(50, 777, torch.float32, 5)
    for ww, bb in ((None, None), (w, None), (None, b)):
        y, stats = T.layer_norm(x, ww, bb)
        check_norm(x, ww, bb, 1e-5, y, stats)
        dx, dw, db = T.layer_norm_backward(dy, x, ww, stats)
        check_norm_back(x, ww, stats, dy, dx, dw, db)
        assert T.layer_norm_backward(dy, x, ww, stats, need_params=False)[1] is None
    y, stats = T.layer_norm(x, w, b)
    dx, dw, db = T.layer_norm_backward(dy, x, w, stats)
    # into pieces of a flat gradient, twice: the sums double, exactly
    flat = torch.zeros(1 + 2 * 777, device="cuda")
    for _ in range(2):
        T.layer_norm_backward(dy, x, w, stats, dw=flat[1:778], db=flat[778:], accumulate=True)
    assert torch.equal(flat[1:778], dw + dw) and torch.equal(flat[778:], db + db) and flat[0] == 0
    # y over x, dx over dy
    for rows, n in ((50, 777), (3, 20000)):
        x, w, b, dy = norm_inputs(rows, n, torch.float32, 6)
        y, stats = T.layer_norm(x, w, b)
        dx, _, _ = T.layer_norm_backward(dy, x, w, stats)
        d2 = dy.clone()
        assert torch.equal(T.layer_norm_backward(d2, x, w, stats, dx=d2)[0], dx)
        x2 = x.clone()
        assert torch.equal(T.layer_norm(x2, w, b, out=x2)[0], y)


@pytest.mark.parametrize("rows,n", [(1, 300), (20, 300), (3, 777), (2, 5000), (4, 9000), (33, 300), (5, 777)])
def test_norm_gradients_add_to_what_is_there(cuda_device, rows, n):
    """Few rows: one block may have them all and write the sums itself."""
    for dtype in (torch.float32, torch.bfloat16):
        x, w, b, dy = norm_inputs(rows, n, dtype, rows + n)
        y, stats = T.layer_norm(x, w, b)
        dx, dw, db = T.layer_norm_backward(dy, x, w, stats)
        check_norm_back(x, w, stats, dy, dx, dw, db)
        flat = torch.full((2 * n + 3,), 0.5, device="cuda")
        T.layer_norm_backward(dy, x, w, stats, dw=flat[1: n + 1], db=flat[n + 2: 2 * n + 2], accumulate=True)
        assert torch.equal(flat[1: n + 1], 0.5 + dw) and torch.equal(flat[n + 2: 2 * n + 2], 0.5 + db)
        assert (flat[[0, n + 1, 2 * n + 2]] == 0.5).all()


def test_norm_repeats_bit_for_bit_and_takes_leading_dimensions(cuda_device):
    x, w, b, dy = norm_inputs(2000, 640, torch.bfloat16, 8)
    y, stats = T.layer_norm(x, w, b)
    first = T.layer_norm_backward(dy, x, w, stats)
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(first, T.layer_norm_backward(dy, x, w, stats)))
    y3, stats3 = T.layer_norm(x.view(20, 100, 640), w, b)
    assert y3.shape == (20, 100, 640) and torch.equal(y3.view(2000, 640), y) and torch.equal(stats3, stats)


def test_norm_of_no_rows_constant_rows_and_values_that_are_not_finite(cuda_device):
    w = torch.ones(96, device="cuda")
    x = torch.empty(0, 96, device="cuda")
    y, stats = T.layer_norm(x, w, w)
    assert y.shape == (0, 96) and stats.shape == (2, 0)
    dx, dw, db = T.layer_norm_backward(x, x, w, stats)
    assert dx.shape == (0, 96) and not dw.any() and not db.any()
    kept = torch.full((96,), 3.0, device="cuda")
    T.layer_norm_backward(x, x, w, stats, dw=kept, db=kept.clone(), accumulate=True)
    assert (kept == 3).all()
    x = torch.full((4, 96), 1.5, device="cuda")
    x[1, 5] = math.inf
    x[2, 7] = math.nan
    x[3] = 2.0
    y, stats = T.layer_norm(x, w, w, 1e-5)
    assert (y[0] == 1).all() and (y[3] == 1).all() and stats[0].tolist()[0] == 1.5
    assert y[1].isnan().all() and y[2].isnan().all()
    dx, dw, _ = T.layer_norm_backward(torch.ones_like(x), x, w, stats)
    assert dx[0].isfinite().all() and dx[1].isnan().all() and dw.isnan().all()
    # large values: the squares of deviations stay finite although x itself is far from zero
    big = 1e4 + torch.randn(3, 4000, generator=gen(1), device="cuda")
    y, stats = T.layer_norm(big, None, None, 1e-5)
    check_norm(big, None, None, 1e-5, y, stats)


def test_norm_gradient_against_differences(cuda_device):
    x, w, b, dy = norm_inputs(6, 37, torch.float32, 9)
    xr, wr, br = x.clone().requires_grad_(), w.clone().requires_grad_(), b.clone().requires_grad_()
    (A.layer_norm(xr, wr, br, 1e-3) * dy).sum().backward()
    f = lambda x, w, b: float((norm64(x, w, b, 1e-3)[0] * dy.double()).sum())  # noqa: E731
    g = gen(3)
    for name, got in (("x", xr.grad), ("w", wr.grad), ("b", br.grad)):
        for _ in range(4):
            d = torch.randn(got.shape, generator=g, device="cuda", dtype=torch.float64)
            args = dict(x=x.double(), w=w.double(), b=b.double())
            step = 1e-5
            up, down = dict(args), dict(args)
            up[name], down[name] = args[name] + step * d, args[name] - step * d
            want = (f(**up) - f(**down)) / (2 * step)
            size = float((got.double() * d).abs().sum())
            # the difference's own error: step^2 and the cancellation of 64-bit values over 2 step
            assert abs(float((got.double() * d).sum()) - want) <= CHAIN * U * size + 1e-7 * size + 1e-6, name


# ---- log probabilities -------------------------------------------------------------------------------


def lp64(z, ids, scale):
    z = z.double() * float(np.float32(scale))     # the operators take it in 32 bits
    m = z.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    e = (z - m).exp()
    s = e.sum(-1, keepdim=True)
    lse = m + s.log()
    # (z - m) - log s, not z - lse: a logit of the format's lowest value absorbs log s even in 64 bits
    logp = torch.where(z == -math.inf, -math.inf, (z - m) - s.log())
    p = logp.exp()
    h = -torch.where(p > 0, p * logp, 0.0).sum(-1)
    inside = (ids >= 0) & (ids < z.shape[1])
    at = logp.gather(1, ids.clamp(0, z.shape[1] - 1).long()[:, None]).squeeze(1)
    return torch.where(inside, at, 0.0), h, lse.squeeze(1), logp, p


def order64(z, k):
    """The k largest of each row, larger first, then the smaller index; NaN above all."""
    zf = torch.where(z.isnan(), math.inf, z.float()) + 0.0
    nan_first = z.isnan().to(torch.int64)
    out = []
    for r in range(z.shape[0]):
        key = sorted(range(z.shape[1]), key=lambda i: (-int(nan_first[r, i]), -float(zf[r, i]), i))[:k]
        out.append(key)
    return torch.tensor(out, dtype=torch.int32)


def check_lp(z, ids, top, scale, r, order=True):
    logp, h, lse, every, p = lp64(z, ids, scale)
    v = z.shape[1]
    chain = v / 256 + 64                       # additions per thread, tree, roundings of the exponent
    fin = torch.isfinite(lse)
    size = torch.where(fin, lse.abs(), 0.0)
    # 2^x is good to 2 units; its argument's rounding enters with the weight of p, within the entropy's size
    rel = chain * U + 4 * U * (h + 4)
    for got, want, tol in ((r.stats[0], logp, rel + 4 * U * torch.where(logp.isfinite(), logp.abs(), 0.0)),
                           (r.stats[1], h, (rel + 4 * U) * (h + 4)), (r.stats[2], lse, rel + 4 * U * size)):
        ok = torch.isfinite(want)
        near(got[ok], want[ok], tol[ok] + 1e-300)
        assert torch.equal(got[~ok].double(), want[~ok])
    if top:
        idx = r.top_idx.long()
        if order:
            assert torch.equal(r.top_idx.cpu(), order64(z.cpu(), top))
        want = every.gather(1, idx)
        ok = torch.isfinite(want)
        near(r.top_logp[ok], want[ok], (rel[:, None] + 4 * U * torch.where(ok, want.abs(), 0.0))[ok], "top")
        assert torch.equal(r.top_logp[~ok].double(), want[~ok])


LP_SIZES = [(1, 1, 1), (3, 5, 5), (2, 33, 32), (7, 300, 3), (4, 2048, 20), (2, 4099, 32), (1, 40000, 20), (1, 131072, 5), (3, 70001, 8),
            (320, 1000, 1), (700, 517, 0), (2, 32000, 0)]


def lp_inputs(rows, v, dtype, seed, spread=2.0):
    g = gen(seed)
    z = (spread * torch.randn(rows, v, generator=g, device="cuda")).to(dtype)
    return z, torch.randint(0, v, (rows,), generator=g, device="cuda")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,v,top", LP_SIZES)
def test_logprobs(cuda_device, rows, v, top, dtype):
    z, ids = lp_inputs(rows, v, dtype, rows + v)
    for scale in (1.0, 0.37):
        check_lp(z, ids, top, scale, T.token_logprobs(z, ids, top=top, scale=scale), order=rows * v <= 300000)
    r = T.token_logprobs(z, ids.to(torch.int32), top=top)
    assert torch.equal(r.stats, T.token_logprobs(z, ids).stats)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("v,pad,offset", [(1000, 24, 8), (1001, 2, 1), (999, 9, 3), (30011, 1, 5), (6, 3, 1)])
def test_logprobs_of_strided_rows(cuda_device, dtype, v, pad, offset):
    z, ids = lp_inputs(5, v, dtype, v)
    zs = strided(z, pad, offset)
    r = T.token_logprobs(zs, ids, top=3)
    check_lp(z, ids, 3, 1.0, r)
    d = torch.randn(5, device="cuda", generator=gen(1))
    a = T.token_logprobs_backward(z, ids, r.lse, d, top_idx=r.top_idx, d_top=r.top_logp)
    for out in (None, strided(z, pad, offset), strided(z, pad + 1, offset + 1)):   # alike and unlike within 16 bytes
        b = T.token_logprobs_backward(zs, ids, r.lse, d, top_idx=r.top_idx, d_top=r.top_logp, out=out)
        assert torch.equal(a, b)
        if out is not None:
            assert (out._base[:offset] == 7).all()
            assert (out.as_strided((4, out.stride(0) - v), out.stride(), out.storage_offset() + v) == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_logprobs_masks(cuda_device, dtype):
    """-inf and the type's lowest value as masks, rows that they leave empty, one finite value, large offsets."""
    low = torch.finfo(dtype).min
    v = 2500
    z, ids = lp_inputs(10, v, dtype, 4)
    z[0, 100:] = -math.inf
    z[1] = -math.inf                          # nothing left
    z[2] = low                                # everything masked with the lowest value: uniform
    z[3, 1:] = low
    z[4] = -math.inf
    z[4, 1777] = 3.0                          # one left
    z[5, ::2] = -math.inf
    z[6, :2049] = -math.inf                   # whole threads see nothing at first
    z[7] = low
    z[7, 5] = -math.inf
    z[8] = torch.where(torch.rand(v, generator=gen(1), device="cuda") < 0.5, low, z[8])
    z[9] += 3000.0 if dtype != torch.float16 else 900.0
    ids = torch.tensor([5, 3, 7, 0, 1777, 0, 2300, 5, -100, v + 3], device="cuda")
    r = T.token_logprobs(z, ids, top=4)
    check_lp(z, ids, 4, 1.0, r)
    assert r.lse[1] == -math.inf and r.entropy[1] == 0 and r.logp[1] == -math.inf and (r.top_logp[1] == -math.inf).all()
    assert r.top_idx[1].tolist() == [0, 1, 2, 3] and r.top_idx[2].tolist() == [0, 1, 2, 3]
    assert r.logp[8] == 0 and r.logp[9] == 0
    g = gen(2)
    d, dh, dt = (torch.randn(s, generator=g, device="cuda") for s in ((10,), (10,), (10, 4)))
    out = T.token_logprobs_backward(z, ids, r.lse, d, entropy=r.entropy, d_entropy=dh, top_idx=r.top_idx, d_top=dt)
    check_lp_back(z, ids, 1.0, r, d, dh, dt, out)


def check_lp_back(z, ids, scale, r, d, dh, dt, out):
    """Against the formula, with the statistics as they were given."""
    rows, v = z.shape
    scale = float(np.float32(scale))
    lse, h = r.lse.double()[:, None], r.entropy.double()[:, None]
    zs = z.double() * scale
    logp = torch.where((zs == -math.inf) | (lse == -math.inf), -math.inf, zs - lse)
    p = logp.exp()
    inside = (ids >= 0) & (ids < v)
    one = torch.zeros_like(p)
    at = torch.where(inside, ids, 0).long()[:, None]
    gl = torch.where(inside, d.double(), 0.0) if d is not None else torch.zeros(rows, device="cuda", dtype=torch.float64)
    one.scatter_add_(1, at, gl[:, None])
    size = torch.zeros_like(p).scatter_add_(1, at, gl.abs()[:, None])
    total = gl.clone()
    if dt is not None:
        one.scatter_add_(1, r.top_idx.long(), dt.double())
        size.scatter_add_(1, r.top_idx.long(), dt.double().abs())
        total = total + dt.double().sum(-1)
    mag = gl.abs() + (dt.double().abs().sum(-1) if dt is not None else 0)
    lp = torch.where(p > 0, logp, 0.0)
    gh = dh.double()[:, None] if dh is not None else torch.zeros_like(lse)
    want = scale * (one - p * (total[:, None] + gh * (lp + h)))
    # p: 2^x to 2 units and the roundings of its argument; the sums over the alternatives: their number
    relp = 8 * U + 4 * U * lp.abs() + 2 * U * torch.where(lse.isfinite(), lse.abs(), 0.0)
    tol = scale * (p * (relp + 40 * U) * (mag[:, None] + gh.abs() * (lp.abs() + h.abs())) + 40 * U * size)
    near(out, want, tol + HALF[z.dtype] * (want.abs() + tol) + TINY[z.dtype] + 1e-37, "dlogits")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,v,top", LP_SIZES)
def test_logprobs_gradient(cuda_device, rows, v, top, dtype):
    z, ids = lp_inputs(rows, v, dtype, rows * 3 + v)
    g = gen(7)
    d, dh, dt = (torch.randn(s, generator=g, device="cuda") for s in ((rows,), (rows,), (rows, top)))
    for scale in (1.0, 1.7):
        r = T.token_logprobs(z, ids, top=top, scale=scale)
        kw = dict(top_idx=r.top_idx, d_top=dt) if top else {}
        out = T.token_logprobs_backward(z, ids, r.lse, d, scale=scale, **kw)
        check_lp_back(z, ids, scale, r, d, None, dt if top else None, out)
        out = T.token_logprobs_backward(z, ids, r.lse, d, entropy=r.entropy, d_entropy=dh, scale=scale, **kw)
        check_lp_back(z, ids, scale, r, d, dh, dt if top else None, out)
        out = T.token_logprobs_backward(z, ids, r.lse, None, entropy=r.entropy, d_entropy=dh, scale=scale)
        check_lp_back(z, ids, scale, r, None, dh, None, out)
        over = z.clone()
        assert torch.equal(T.token_logprobs_backward(over, ids, r.lse, None, entropy=r.entropy, d_entropy=dh, scale=scale, out=over), out)
        over = z.clone()
        a = T.token_logprobs_backward(z, ids, r.lse, d, scale=scale, **kw)
        assert torch.equal(T.token_logprobs_backward(over, ids, r.lse, d, scale=scale, out=over, **kw), a)


def test_logprobs_alternatives_of_equal_rising_and_not_finite_logits(cuda_device):
    for dtype in TYPES:
        for rows, v in ((2, 3000), (1, 90001), (400, 700)):
            ids = torch.zeros(rows, dtype=torch.int64, device="cuda")
            z = torch.full((rows, v), 1.25, dtype=dtype, device="cuda")
            assert (T.token_logprobs(z, ids, top=32).top_idx.cpu() == torch.arange(32)).all()
            z = (torch.arange(v, device="cuda") // 7).to(dtype).expand(rows, v).contiguous() / 64     # rising, with ties
            r = T.token_logprobs(z, ids, top=32)
            assert torch.equal(r.top_idx.cpu(), order64(z[:1].cpu(), 32).expand(rows, 32))
            z = z.flip(1).contiguous()
            r = T.token_logprobs(z, ids, top=32)
            assert torch.equal(r.top_idx.cpu(), order64(z[:1].cpu(), 32).expand(rows, 32))
    z, ids = lp_inputs(4, 5000, torch.float32, 3)
    z[0, 17], z[0, 4000] = math.nan, -math.nan
    z[1, 900] = math.inf
    z[2, 100], z[2, 50], z[2, 3000] = 0.0, -0.0, 0.0
    z[2, :40] = -1.0
    z[2] = torch.where(z[2] > 0, -z[2], z[2])
    r = T.token_logprobs(z, ids, top=3)
    assert torch.equal(r.top_idx.cpu(), order64(z.cpu(), 3))
    assert r.top_idx[2].tolist() == [50, 100, 3000] and r.top_idx[0].tolist()[:2] == [17, 4000] and r.top_idx[1, 0] == 900
    assert r.stats[:, 0].isnan().all() and r.stats[1:, 1].isnan().all()
    assert r.stats[:, 2:].isfinite().all()


def test_logprobs_of_rows_with_many_batches(cuda_device):
    """Enough rows that one CTA has each, long enough that several batches share one of the maxima it keeps."""
    for dtype, v in ((torch.float32, 200003), (torch.bfloat16, 300001)):
        z, ids = lp_inputs(600, v, dtype, 17)
        r = T.token_logprobs(z, ids, top=7)
        for rows in (slice(0, 40), slice(590, 600)):
            part = T.TokenLogprobs(r.stats[:, rows], r.top_idx[rows], r.top_logp[rows])
            check_lp(z[rows], ids[rows], 7, 1.0, part, order=False)
        order = z[:40].float().sort(dim=1, descending=True, stable=True).indices[:, :7]
        assert torch.equal(r.top_idx[:40].long(), order)
        assert torch.equal(z.gather(1, r.top_idx.long()), z.topk(7, dim=1).values)


def test_logprobs_gradient_against_differences(cuda_device):
    z, ids = lp_inputs(3, 41, torch.float32, 12)
    zr = z.clone().requires_grad_()
    logp, h, _, idx, top = A.token_logprobs(zr, ids, top=4, scale=0.8)
    g = gen(5)
    a, b, c = (torch.randn(s, generator=g, device="cuda", dtype=torch.float64) for s in ((3,), (3,), (3, 4)))
    ((logp * a).sum() + (h * b).sum() + (top * c).sum()).backward()

    def f(z):
        lp, hh, _, every, _ = lp64(z, ids, 0.8)
        return float((lp * a).sum() + (hh * b).sum() + (every.gather(1, idx.long()) * c).sum())

    for _ in range(6):
        d = torch.randn(z.shape, generator=g, device="cuda", dtype=torch.float64)
        step = 1e-5
        want = (f(z.double() + step * d) - f(z.double() - step * d)) / (2 * step)
        size = float((zr.grad.double() * d).abs().sum())
        assert abs(float((zr.grad.double() * d).sum()) - want) <= CHAIN * U * size + 1e-7 * size + 1e-6


def test_logprobs_of_no_rows(cuda_device):
    z = torch.empty(0, 50, device="cuda")
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    r = T.token_logprobs(z, ids, top=2)
    assert r.stats.shape == (3, 0) and r.top_idx.shape == (0, 2)
    assert T.token_logprobs_backward(z, ids, r.lse, r.logp).shape == (0, 50)


# ---- AdamW -------------------------------------------------------------------------------------------

HYPER = dict(lr=1e-2, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)


def adamw64(p, g, m, v, t, lr=1e-2, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1):
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    upd = (m / (1 - betas[0] ** t)) / ((v / (1 - betas[1] ** t)).sqrt() + eps)
    return p * (1 - lr * weight_decay) - lr * upd, m, v, lr * upd


def check_f32(opt, before, grads, t, scale=1.0):
    for i, (p0, m0, v0) in enumerate(before):
        if grads[i] is None:
            assert torch.equal(opt.params[i], p0) and torch.equal(opt.m[i], m0) and torch.equal(opt.v[i], v0)
            continue
        g = grads[i].double() * scale
        p1, m1, v1, upd = adamw64(p0.double(), g, m0.double(), v0.double(), t)
        tol = 8 * U * (m0.double().abs() + g.abs())
        near(opt.m[i], m1, tol, f"m[{i}]")
        near(opt.v[i], v1, 8 * U * (v0.double() + g * g), f"v[{i}]")
        # the update carries m's absolute error, which cancellation can leave large beside m itself
        slack = tol / (m1.abs() + 1e-300) * upd.abs()
        tol_p = 8 * U * p0.double().abs() + 32 * U * upd.abs() + torch.where(m1 == 0, 0.0, slack)
        near(opt.params[i], p1, tol_p + HALF[opt.params[i].dtype] * (p1.abs() + tol_p) + 1e-300, f"p[{i}]")
        if opt.copies is not None:
            assert torch.equal(opt.copies[i], opt.params[i].to(opt.copies[i].dtype))


def cut(flat, sizes, gap=0):
    out, at = [], 0
    for n in sizes:
        out.append(flat[at: at + n])
        at += n + gap
    return out


SIZES = [1, 3, 0, 255, 256, 257, 4096, 5003, 8, 2047, 2049, 100000]


@pytest.mark.parametrize("gdtype", TYPES)
@pytest.mark.parametrize("pdtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gaps", [(0, 0), (1, 2), (4, 4)])
def test_adamw_f32_states(cuda_device, pdtype, gdtype, gaps):
    g = gen(1)
    total = sum(SIZES) + 64 * len(SIZES)
    rnd = lambda dt: torch.randn(total, generator=g, device="cuda").to(dt)  # noqa: E731
    # views of flat vectors: with different gaps their addresses have no common alignment
    params = cut(rnd(pdtype), SIZES, gaps[0])
    m, v = cut(rnd(torch.float32) * 0.1, SIZES, gaps[0]), cut(rnd(torch.float32).square(), SIZES, gaps[0])
    copies = cut(rnd(torch.bfloat16 if gaps[0] else torch.float16), SIZES, gaps[1]) if pdtype == torch.float32 else None
    opt = T.AdamW(params, m=m, v=v, copies=copies, step_count=4, **HYPER)
    for t in (5, 6):
        grads = cut(rnd(gdtype), SIZES, gaps[1])
        if t == 6:
            grads[3] = grads[7] = None
        before = [(p.clone(), a.clone(), b.clone()) for p, a, b in zip(params, m, v)]
        scale = torch.tensor([0.25], device="cuda") if t == 6 else None
        opt.step(grads, grad_scale=scale)
        assert opt.step_count == t
        check_f32(opt, before, grads, t, 0.25 if t == 6 else 1.0)


def test_adamw_touches_nothing_else_and_takes_many_tensors(cuda_device):
    sizes = [(i * 37) % 300 + 1 for i in range(900)]
    flat = torch.full((sum(s + 3 for s in sizes),), 5.0, device="cuda")
    params = cut(flat, sizes, 3)
    opt = T.AdamW(params, **HYPER)
    grads = [torch.randn(s, generator=gen(s), device="cuda") for s in sizes]
    before = [(p.clone(), a.clone(), b.clone()) for p, a, b in zip(params, opt.m, opt.v)]
    opt.step(grads)
    check_f32(opt, before, grads, 1)
    inside = torch.zeros_like(flat, dtype=torch.bool)
    for c in cut(inside, sizes, 3):
        c[:] = True
    assert (flat[~inside] == 5).all()


def mix(x):
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def words(seed, tensor, n, start=0):
    key = mix((mix(mix(seed & 0xFFFFFFFF) ^ (seed >> 32)) + tensor) & 0xFFFFFFFF)
    i = np.arange(start, start + n, dtype=np.int64)
    return mix((i & 0xFFFFFFFF) ^ ((i >> 32) * 0x9E3779B9 & 0xFFFFFFFF) ^ key)


def blocks_of(x):
    n = x.numel()
    nb = -(-n // 256)
    return torch.nn.functional.pad(x, (0, nb * 256 - n)).view(nb, 256)


def unit_of(y):
    """One unit of the last place of an e4m3 number of magnitude y."""
    return torch.exp2(torch.floor(torch.log2(y.clamp_min(2.0 ** -6))) - 3)


def check_8bit(opt, before, grads, t, seed, start=0):
    for i, (p0, m0, v0, ms0, vs0) in enumerate(before):
        n = p0.numel()
        if n == 0:
            continue
        spread = lambda s: s.double().repeat_interleave(256)[:n]  # noqa: E731
        g = grads[i].double()
        p1, m1, v1, upd = adamw64(p0.double(), g, m0.double() * spread(ms0), (v0.double() * spread(vs0)) ** 2, t)
        r1 = v1.sqrt()
        cancel = 16 * U * (g.abs() + m0.double().abs() * spread(ms0))
        if opt.params[i].dtype == torch.float32:
            slack = torch.where(m1 == 0, 0.0, cancel / (m1.abs() + 1e-300) * upd.abs())
            near(opt.params[i], p1, 8 * U * p0.double().abs() + 32 * U * upd.abs() + slack + 1e-300, "p")
        else:
            # rounded up or down from p1: within one unit of the last place
            ulp = 2.0 ** -7 * torch.exp2(torch.floor(torch.log2(p1.abs().clamp_min(1e-30))))
            near(opt.params[i], p1, ulp * (1 + 1e-3) * (1.0 if seed is not None else 0.5) + 32 * U * upd.abs() + 1e-300, "p")
        w = words(seed, i, n, start) if seed is not None else None
        for got, scale, want, shift in ((opt.m[i], opt.m_scale[i], m1, 0), (opt.v[i], opt.v_scale[i], r1, 16)):
            amax = blocks_of(want.abs()).amax(1)
            near(scale, amax / 448, 32 * U * amax / 448 + blocks_of(cancel).amax(1) / 448 + 1e-300, "scale")
            s = spread(scale)
            y = torch.where(s > 0, want.abs() / s.clamp_min(1e-300), 0.0)
            unit = unit_of(y)
            u = torch.from_numpy(((w >> shift) & 0xFFFF).astype(np.float64)).cuda() * 2.0 ** -16 + 2.0 ** -17 if w is not None else 0.5
            x = y / unit + u
            code = torch.floor(x) * unit
            if shift:
                code = torch.where(want > 0, code.clamp_min(2.0 ** -9), code)
            code = code.clamp_max(448.0)
            # where y / unit + u is within the error of fp32 of a whole number the other neighbour is right as well
            close = ((x - torch.round(x)).abs() <= 64 * U * (y / unit + 1) + cancel / (s.clamp_min(1e-300) * unit)) | (y >= 447.9)
            diff = (got.double().abs() - code).abs()
            assert (diff[~close] == 0).all(), f"{int((diff[~close] > 0).sum())} codes"
            assert (diff[close] <= 2.01 * unit[close]).all()
            # dither of 16 bits: 64-bit and 32-bit arithmetic seldom part
            assert float(close.double().mean()) < 0.01 or n < 3000
            signed = got.double() * want < 0
            assert not signed[y > unit].any()
        if opt.copies is not None:
            assert torch.equal(opt.copies[i], opt.params[i].to(opt.copies[i].dtype))


@pytest.mark.parametrize("gdtype", TYPES)
@pytest.mark.parametrize("pdtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gap", [0, 1, 8])
def test_adamw_8bit_states(cuda_device, pdtype, gdtype, gap):
    g = gen(2)
    sizes = [8 * s if gap == 8 else s for s in SIZES]        # every tensor aligned, or hardly one
    total = sum(sizes) + 64 * len(sizes)
    params = cut(torch.randn(total, generator=g, device="cuda").to(pdtype), sizes, gap)
    copies = cut(torch.zeros(total, device="cuda", dtype=torch.bfloat16), sizes, gap) if pdtype == torch.float32 else None
    opt = T.AdamW(params, state="e4m3", copies=copies, **HYPER)
    for t, seed in ((1, 11), (2, 1 << 40 | 5), (3, None), (4, 2 ** 64 - 1)):
        grads = cut((torch.randn(total, generator=g, device="cuda") * torch.exp2(-torch.arange(total, device="cuda") % 12)).to(gdtype),
                    sizes, gap)
        before = [(p.clone(), a.clone(), b.clone(), c.clone(), d.clone())
                  for p, a, b, c, d in zip(params, opt.m, opt.v, opt.m_scale, opt.v_scale)]
        opt.step(grads, seed=seed)
        check_8bit(opt, before, grads, t, seed)


def test_adamw_8bit_does_not_depend_on_how_it_is_divided(cuda_device):
    """With a large tensor behind them the others' blocks are dealt out differently: the same bits come out."""
    g = gen(9)
    sizes = [5003, 256, 70001, 1 << 16]
    big = 12_000_011
    p = [torch.randn(n, generator=g, device="cuda").to(torch.bfloat16) for n in sizes + [big]]
    q = [t.clone() for t in p]
    a, b = T.AdamW(p, state="e4m3", **HYPER), T.AdamW(q[:-1], state="e4m3", **HYPER)
    for t in (1, 2):
        grads = [(torch.randn(n, generator=g, device="cuda") * 1e-3).to(torch.bfloat16) for n in sizes + [big]]
        a.step(grads, seed=t)
        b.step(grads[:-1], seed=t)
    for x, y in zip((p, a.m, a.v, a.m_scale, a.v_scale), (q, b.m, b.v, b.m_scale, b.v_scale)):
        assert all(torch.equal(i.float(), j.float()) for i, j in zip(x[:-1], y[: len(sizes)]))
    last = T.AdamW([p[-1]], state="e4m3", m=[a.m[-1]], v=[a.v[-1]], m_scale=[a.m_scale[-1]], v_scale=[a.v_scale[-1]], step_count=2, **HYPER)
    before = [(p[-1].clone(), a.m[-1].clone(), a.v[-1].clone(), a.m_scale[-1].clone(), a.v_scale[-1].clone())]
    grads = [(torch.randn(big, generator=g, device="cuda") * 1e-3).to(torch.bfloat16)]
    last.step(grads, seed=77)
    check_8bit(last, before, grads, 3, 77)


def test_offsets_beyond_32_bits(cuda_device):
    """Rows 2^31 elements apart, and a tensor of more than 2^32 elements."""
    far = (1 << 31) + 8
    buf = torch.zeros(2 * far + 4096, dtype=torch.bfloat16, device="cuda")
    x, w, b, dy = norm_inputs(3, 1024, torch.bfloat16, 2)
    xs, out = buf.as_strided((3, 1024), (far, 1)), buf.as_strided((3, 1024), (far, 1), 2048)
    xs.copy_(x)
    y, stats = T.layer_norm(xs, w, b, out=out)
    check_norm(x, w, b, 1e-5, y, stats)
    dx, dw, db = T.layer_norm_backward(dy, xs, w, stats, dx=out)
    check_norm_back(x, w, stats, dy, dx, dw, db)
    ids = torch.tensor([3, 500, 1023], device="cuda")
    r = T.token_logprobs(xs, ids, top=3)
    check_lp(x, ids, 3, 1.0, r)
    d = torch.ones(3, device="cuda")
    check_lp_back(x, ids, 1.0, r, d, None, None, T.token_logprobs_backward(xs, ids, r.lse, d, out=out))
    del xs, out, buf
    n = (1 << 32) + 777
    p, g = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    start, gg = (1 << 32) - 1024, gen(6)
    for t in (p, g):
        t[start:] = torch.randn(n - start, generator=gg, device="cuda").to(torch.bfloat16)
    opt = T.AdamW([p], state="e4m3", **HYPER)
    tail = T.AdamW.__new__(T.AdamW)                    # the same step, seen from `start` on
    tail.params, tail.m, tail.v, tail.copies = [p[start:]], [opt.m[0][start:]], [opt.v[0][start:]], None
    tail.m_scale, tail.v_scale = [opt.m_scale[0][start // 256:]], [opt.v_scale[0][start // 256:]]
    for t in (1, 2):
        before = [tuple(x[0].clone() for x in (tail.params, tail.m, tail.v, tail.m_scale, tail.v_scale))]
        opt.step([g], seed=40 + t)
        check_8bit(tail, before, [g[start:]], t, 40 + t, start)
    assert not p[:start].any() and not opt.m[0][:4096].float().any()


def test_adamw_8bit_is_right_on_average_and_moves_slowly(cuda_device):
    """Stochastic rounding: the mean error over many elements vanishes, and a second moment that shrinks by a thousandth
    a step does shrink."""
    n = 1 << 20
    g = torch.rand(n, generator=gen(4), device="cuda") * 0.1 + 0.01
    opt = T.AdamW([torch.zeros(n, device="cuda")], state="e4m3", betas=(0.9, 0.999), lr=0.0)
    opt.step([g], seed=1)
    scale = lambda s: s[0].double().repeat_interleave(256)  # noqa: E731
    for got, want in ((opt.m[0].double() * scale(opt.m_scale), 0.1 * g.double()),
                      (opt.v[0].double() * scale(opt.v_scale), math.sqrt(0.001) * g.double())):
        # an error is at most a unit, an eighth of the value: standard deviation below an eighth / 2 of it
        bound = 6 * 0.0625 / math.sqrt(n)
        assert abs(float(((got - want) / want).mean())) < bound
    v0 = float((opt.v[0].double() * scale(opt.v_scale)).square().mean())
    for t in range(200):
        opt.step([torch.zeros_like(g)], seed=100 + t)
    v1 = float((opt.v[0].double() * scale(opt.v_scale)).square().mean())
    # each rounding adds its variance to the square: at most (unit / 2)^2 = (value / 16)^2 a step; without dither it stays at v0
    assert v0 * 0.999 ** 200 * 0.95 < v1 < v0


def test_adamw_values_that_are_not_finite_stay_alone(cuda_device):
    for state, n in (("f32", 5000), ("e4m3", 5000), ("e4m3", 4096)):
        p = torch.ones(n, device="cuda")
        opt = T.AdamW([p], state=state, **HYPER)
        g = torch.randn(n, generator=gen(1), device="cuda")
        g[3], g[777], g[4000] = math.nan, math.inf, -math.inf
        for t in range(2):
            opt.step([g], seed=t)
        bad = torch.zeros(n, dtype=torch.bool, device="cuda")
        bad[[3, 777, 4000]] = True
        for q in (opt.m[0].float(), opt.v[0].float()):
            assert not q[bad].isfinite().any() and q[~bad].isfinite().all()
        assert p[~bad].isfinite().all() and not p[3].isfinite()
        if state == "e4m3":
            assert opt.m_scale[0].isfinite().all() and opt.v_scale[0].isfinite().all()
    # bfloat16 parameters, rounded stochastically: infinities and NaN stay what they are
    p = torch.tensor([math.inf, -math.inf, math.nan, 1.0], device="cuda").to(torch.bfloat16)
    T.AdamW([p], state="f32", lr=0.0).step([torch.zeros(4, device="cuda")], seed=3)
    assert p[0] == math.inf and p[1] == -math.inf and p[2].isnan() and p[3] == 1


def test_adamw_follows_its_parameters_and_refuses_what_does_not_fit(cuda_device):
    g = gen(3)
    p = [torch.randn(n, generator=g, device="cuda") for n in (1000, 7)]
    q = [t.clone() for t in p]
    grads = [torch.randn(n, generator=g, device="cuda") for n in (1000, 7)]
    a, b = T.AdamW(p, **HYPER), T.AdamW(q, **HYPER)
    a.step(grads)
    p[0].data = p[0].data.clone()                      # other storage: the step goes where the parameter is now
    version = p[0]._version
    a.step(grads)
    assert p[0]._version > version                     # autograd is told
    b.step(grads)
    b.step(grads)
    assert all(torch.equal(x, y) for x, y in zip(p, q))
    for bad in ([grads[0]], [grads[0], grads[0]], [grads[0].double(), grads[1]], [grads[0], grads[1].half()], [grads[0].cpu(), grads[1]],
                [torch.randn(2000, device="cuda")[::2], grads[1]], "xy"):
        with pytest.raises((TypeError, ValueError), match="grads"):
            a.step(bad)
    with pytest.raises(TypeError, match="grad_scale"):
        a.step(grads, grad_scale=torch.ones(2, device="cuda"))
    assert a.step_count == 2 and all(torch.equal(x, y) for x, y in zip(p, q))
    a.params.append(p[0])
    with pytest.raises(ValueError, match="params"):
        a.step(grads)


def test_bindings_refuse_what_the_kernels_could_not_read(cuda_device):
    x, w, b, dy = norm_inputs(8, 64, torch.float32, 1)
    z, ids = lp_inputs(8, 64, torch.float32, 1)
    y, stats = T.layer_norm(x, w, b)
    r = T.token_logprobs(z, ids, top=2)
    wide = torch.zeros(8, 128, device="cuda")
    for call in (lambda: T.layer_norm(wide[:, ::2], w, b), lambda: T.layer_norm(x, w[:32], b), lambda: T.layer_norm(x, w, b.cpu()),
                 lambda: T.layer_norm(x[:1].expand(8, 64), w, b), lambda: T.layer_norm(x.double()), lambda: T.layer_norm(x, out=x.half()),
                 lambda: T.layer_norm(torch.zeros(4, 8, 64, device="cuda").transpose(0, 1)),
                 lambda: T.layer_norm_backward(dy.half(), x, w, stats), lambda: T.layer_norm_backward(dy, x, w, stats[:1]),
                 lambda: T.layer_norm_backward(dy, x, w, stats, dw=torch.zeros(63, device="cuda")),
                 lambda: T.token_logprobs(z[0], ids), lambda: T.token_logprobs(z, ids[:4]), lambda: T.token_logprobs(z, ids.float()),
                 lambda: T.token_logprobs_backward(z, ids, r.lse[:4], r.logp),
                 lambda: T.token_logprobs_backward(z, ids, r.lse, r.logp, top_idx=r.top_idx.long(), d_top=r.top_logp),
                 lambda: T.token_logprobs_backward(z, ids, r.lse, r.logp, out=z.half())):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        T.token_logprobs_backward(z, ids, r.lse, r.logp, top_idx=r.top_idx)
    with pytest.raises(ValueError):
        T.token_logprobs_backward(z, ids, r.lse, r.logp, d_entropy=r.entropy)
    with pytest.raises(ValueError):
        T.layer_norm_backward(dy, x, w, stats, accumulate=True)
    for call, code in ((lambda: T.token_logprobs(z, ids, top=33), S.ETOOBIG), (lambda: T.token_logprobs(z, ids, scale=0.0), S.EINVAL),
                       (lambda: T.layer_norm(x, w.half(), b.half()), S.EINVAL), (lambda: T.layer_norm(x, eps=-1.0), S.EINVAL)):
        with pytest.raises(S.SsgdError) as e:
            call()
        assert e.value.code == code


def test_operators_on_another_stream_and_in_a_graph(cuda_device):
    x, w, b, dy = norm_inputs(300, 512, torch.bfloat16, 3)
    z, ids = lp_inputs(1, 100000, torch.bfloat16, 3)
    p = torch.ones(3000, device="cuda")
    opt = T.AdamW([p], **HYPER)
    grad = torch.randn(3000, generator=gen(1), device="cuda")

    def everything():
        y, stats = T.layer_norm(x, w, b)
        dx, dw, db = T.layer_norm_backward(dy, x, w, stats)
        r = T.token_logprobs(z, ids, top=5)
        dz = T.token_logprobs_backward(z, ids, r.lse, r.logp)
        return [y, stats, dx, dw, db, r.stats, r.top_idx, dz]

    want = everything()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = everything()
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(want, got))
    q = p.clone()
    again = T.AdamW([q], **HYPER)
    again.step([grad])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = everything()
        opt.step([grad])
    for t in got:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(want, got)) and torch.equal(p, q)


def test_autograd_wrappers_match_the_operators(cuda_device):
    x, w, b, dy = norm_inputs(64, 384, torch.bfloat16, 6, torch.bfloat16)
    xr, wr, br = (t.clone().requires_grad_() for t in (x, w, b))
    y = A.layer_norm(xr.view(8, 8, 384), wr, br)
    y.backward(dy.view(8, 8, 384))
    y2, stats = T.layer_norm(x, w, b)
    dx, dw, db = T.layer_norm_backward(dy, x, w, stats)
    assert torch.equal(y.view(64, 384), y2) and torch.equal(xr.grad, dx)
    assert torch.equal(wr.grad, dw.to(w.dtype)) and torch.equal(br.grad, db.to(b.dtype))
    z, ids = lp_inputs(30, 500, torch.float32, 6)
    zr = z.clone().requires_grad_()
    logp, _, _, _, _ = A.token_logprobs(zr, ids)
    (-logp.mean()).backward()
    zt = z.clone().requires_grad_()
    torch.nn.functional.cross_entropy(zt, ids).backward()
    assert (zr.grad - zt.grad).abs().max() <= 1e-6
