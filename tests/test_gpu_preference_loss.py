"""The preference loss and its gradient against the formula in 64 bits.

Tolerances: every difference logp - ref_logp is rounded once (U = 2^-24), the sums are taken in more than 48 bits, x is rounded to fp32, and
the loss and its slope are a few fp32 operations: their own 16 U, and what the error of x does through the first and second derivative."""
import math

import numpy as np
import pytest
import torch

from paper_1903_04488_b200 import autograd as A
from paper_1903_04488_b200 import train_ops as T

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def inputs(lens, seed, before=0, behind=0, noise=0.3, dtype=torch.int32):
    g = gen(seed)
    ends = np.concatenate([[before], before + np.cumsum(np.array(lens, dtype=np.int64))])
    n = int(ends[-1]) + behind
    logp = -3 * torch.rand(n, generator=g, device="cuda")
    ref = logp + noise * torch.randn(n, generator=g, device="cuda")
    return logp, ref, torch.tensor(ends, dtype=dtype, device="cuda")


def formula(logp, ref, starts, beta=0.1, label_smoothing=0.0, kind="sigmoid", average=False, weights=None):
    """loss, rewards, d_logp and a tolerance for each"""
    beta, e = float(np.float32(beta)), float(np.float32(label_smoothing))
    at = starts.long().tolist()
    seqs = len(at) - 1
    diff = logp.double() - (ref.double() if ref is not None else 0.0)
    lens = torch.tensor([b - a for a, b in zip(at, at[1:])], dtype=torch.float64, device="cuda")
    D, size = ([torch.zeros((), dtype=torch.float64, device="cuda") for _ in range(seqs)] for _ in range(2))
    for s, (a, b) in enumerate(zip(at, at[1:])):
        if b > a:
            D[s], size[s] = diff[a:b].sum(), diff[a:b].abs().sum()
    D, size = (torch.stack(x) if x else torch.zeros(0, dtype=torch.float64, device="cuda") for x in (D, size))
    f = torch.where(lens > 0, 1 / lens.clamp_min(1), 0.0) if average else torch.ones_like(lens)
    D, size = (D * f).view(-1, 2), (size * f).view(-1, 2)
    x = beta * (D[:, 0] - D[:, 1])
    dx = beta * U * size.sum(1) + 2 * U * x.abs()
    w = torch.ones_like(x) if weights is None else weights.double()
    if kind == "sigmoid":
        loss = -(1 - e) * torch.nn.functional.logsigmoid(x) - e * torch.nn.functional.logsigmoid(-x)
        slope, second = e - torch.sigmoid(-x), 0.25
    elif kind == "ipo":
        loss, slope, second = ((x - 0.5) / beta) ** 2, 2 * (x - 0.5) / beta ** 2, 2 / beta ** 2
    else:
        loss, slope, second = (1 - x).clamp_min(0), torch.where(x < 1, -1.0, 0.0).double(), 0.0
    live = w != 0
    t_loss = w.abs() * (slope.abs() * dx + second * dx ** 2 + 16 * U * (loss + x.abs() + 1))
    t_slope = (w * beta).abs() * (second * dx + 16 * U * (slope.abs() + 0.1))
    loss, slope = torch.where(live, w * loss, 0.0), torch.where(live, w * beta * slope, 0.0)
    d, t_d = torch.zeros(logp.numel(), dtype=torch.float64, device="cuda"), torch.zeros(logp.numel(), dtype=torch.float64, device="cuda")
    for s, (a, b) in enumerate(zip(at, at[1:])):
        d[a:b] = (slope if s % 2 == 0 else -slope)[s // 2] * f[s]
        t_d[a:b] = t_slope[s // 2] * f[s] + 4 * U * d[a:b].abs()
    return loss, beta * D.t(), d, t_loss, beta * U * size.t() + 4 * U * beta * D.t().abs(), t_d


def check(logp, ref, starts, r, **kw):
    loss, rewards, d, t_loss, t_rewards, t_d = formula(logp, ref, starts, **kw)
    for got, want, tol, name in ((r.loss, loss, t_loss, "loss"), (r.rewards, rewards, t_rewards, "rewards"), (r.d_logp, d, t_d, "d_logp")):
        if got is not None:
            bad = (got.double() - want).abs() > tol + 1e-37
            assert not bad.any(), f"{name}: {int(bad.sum())} outside"


def lengths(pairs, mean, seed):
    rng = np.random.default_rng(seed)
    return [int(x) for x in np.minimum(rng.exponential(mean, 2 * pairs), 20 * mean) * (rng.random(2 * pairs) > 0.1)]


CASES = [([1, 1], 0, 0), ([0, 0], 3, 2), ([5, 0], 0, 0), ([0, 7], 0, 1), ([4096, 4096], 0, 0), ([4095, 1, 1, 4095], 0, 5), ([1] * 400, 0, 0),
         ([0] * 300 + [1, 2] + [0] * 300, 1, 1), ([20000, 3], 0, 0), ([3, 1200000], 7, 9), (lengths(8, 100, 1), 0, 40), (lengths(500, 30, 2), 5000, 9000),
         (lengths(3, 30000, 3), 0, 0), (lengths(4000, 3, 4), 0, 0), ([16] * 6000, 100, 0),
         ([8192, 8192], 0, 0), ([8191, 1, 1, 8191], 0, 3), ([8192, 0, 0, 8192], 0, 0), ([128] * 256, 0, 0), ([100] * 64 + [0] * 2000, 3, 3)]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_preference_loss(cuda_device, case):
    lens, before, behind = CASES[case]
    logp, ref, starts = inputs(lens, case, before, behind)
    pairs = len(lens) // 2
    w = torch.randn(pairs, device="cuda", generator=gen(case))
    for kw in (dict(), dict(label_smoothing=0.1, weights=w), dict(average=True, beta=2.0), dict(kind="ipo", weights=w), dict(kind="hinge", beta=0.3)):
        r = T.preference_loss(logp, ref, starts, **kw)
        check(logp, ref, starts, r, **kw)
        again = T.preference_loss(logp, ref, starts.to(torch.int64), **kw)
        assert all(torch.equal(a, b) for a, b in ((r.loss, again.loss), (r.rewards, again.rewards), (r.d_logp, again.d_logp)))
    r = T.preference_loss(logp, None, starts, need_grad=False)
    assert r.d_logp is None
    check(logp, None, starts, r)
    over = logp.clone()
    assert torch.equal(T.preference_loss(over, ref, starts, out=over).d_logp, T.preference_loss(logp, ref, starts).d_logp)


@pytest.mark.parametrize("offset", [1, 2, 3])
def test_preference_loss_of_tensors_that_lie_anywhere(cuda_device, offset):
    logp, ref, starts = inputs(lengths(40, 300, 5), 5, 10, 20)
    n = logp.numel()
    shift = lambda t, k: torch.cat([t.new_full((k,), 7.0), t, t.new_full((3,), 7.0)])[k: k + t.numel()]  # noqa: E731
    want = T.preference_loss(logp, ref, starts)
    out = shift(logp, 4 - offset)
    got = T.preference_loss(shift(logp, offset), shift(ref, offset + 1), starts, out=out)
    assert torch.equal(got.d_logp, want.d_logp) and torch.equal(got.loss, want.loss)
    assert (out._base[: 4 - offset] == 7).all() and (out._base[4 - offset + n:] == 7).all()


def test_preference_loss_of_what_is_not_finite_stays_in_its_pair(cuda_device):
    """Masks of the lowest number, infinities and NaN in some sequences leave the others as they are, in the same piece of work or not."""
    for lens in ([50] * 40, [3] * 400, [3000] * 12):
        logp, ref, starts = inputs(lens, 6)
        at = starts.tolist()
        logp[at[4]] = -math.inf                # pair 2: cannot be preferred any more
        logp[at[7]] = torch.finfo(torch.float32).min
        logp[at[9]], ref[at[9]] = torch.finfo(torch.float32).min, torch.finfo(torch.float32).min
        logp[at[10]] = math.nan
        r = T.preference_loss(logp, ref, starts)
        assert r.loss[2] == math.inf and (r.d_logp[at[4]: at[5]] == -np.float32(0.1)).all() and (r.d_logp[at[5]: at[6]] == np.float32(0.1)).all()
        assert r.loss[3] == 0 and (r.d_logp[at[6]: at[8]] == 0).all()
        assert r.loss[5].isnan() and r.d_logp[at[10]: at[12]].isnan().all()
        clean, cref = logp.clone(), ref.clone()
        for p in (2, 3, 5):
            clean[at[2 * p]: at[2 * p + 2]] = cref[at[2 * p]: at[2 * p + 2]] = 0
        clean[at[9]] = cref[at[9]] = 0
        c = T.preference_loss(clean, cref, starts)
        rest = [p for p in range(len(lens) // 2) if p not in (2, 3, 5)]
        assert torch.equal(r.loss[rest], c.loss[rest])
        check(clean, cref, starts, c)
        w = torch.ones(len(lens) // 2, device="cuda")
        w[[2, 3, 5]] = 0
        z = T.preference_loss(logp, ref, starts, weights=w)
        assert (z.loss[[2, 3, 5]] == 0).all() and z.d_logp.isfinite().all()


def test_preference_loss_of_nothing_and_of_starts_beyond_the_tokens(cuda_device):
    e = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
    r = T.preference_loss(e(0), e(0), torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert r.loss.numel() == 0 and r.d_logp.numel() == 0
    r = T.preference_loss(e(0), None, torch.zeros(5, dtype=torch.int64, device="cuda"))
    assert torch.allclose(r.loss, torch.full((2,), math.log(2.0), device="cuda")) and (r.rewards == 0).all()
    logp, ref, _ = inputs([9000, 1000], 1)
    r = T.preference_loss(logp, ref, torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert (r.d_logp == 0).all()
    # starts outside the tokens count as the nearest of these
    a = T.preference_loss(logp, ref, torch.tensor([-5, 4000, 1 << 40], device="cuda"))
    b = T.preference_loss(logp, ref, torch.tensor([0, 4000, 10000], device="cuda"))
    assert torch.equal(a.loss, b.loss) and torch.equal(a.d_logp, b.d_logp)


def test_preference_loss_of_more_tokens_than_32_bits_count(cuda_device):
    n = (1 << 30) + 5
    logp = torch.zeros(n, device="cuda")
    cuts = [0, 1 << 29, (1 << 30) - 3, (1 << 30) - 1, n - 2]
    for a, b, v in zip(cuts, cuts[1:], (-2.0 ** -20, -2.0 ** -21, -1.0, -0.5)):      # powers of two: every sum is exact
        logp[a:b] = v
    starts = torch.tensor(cuts, device="cuda")
    r = T.preference_loss(logp, None, starts, beta=0.01)
    D = [(b - a) * v for a, b, v in zip(cuts, cuts[1:], (-2.0 ** -20, -2.0 ** -21, -1.0, -0.5))]
    want = torch.tensor(D, dtype=torch.float64).view(2, 2) * float(np.float32(0.01))
    assert (r.rewards.cpu().double().t() - want).abs().max() <= 2 * U * want.abs().max()
    x = want[:, 0] - want[:, 1]
    slope = -torch.sigmoid(-x) * float(np.float32(0.01))
    for a, b, v in zip(cuts, cuts[1:], (slope[0], -slope[0], slope[1], -slope[1])):
        piece = r.d_logp[a:b]
        assert float(piece.min()) == float(piece.max()) and abs(float(piece[0]) - float(v)) <= 64 * U * 0.01
    assert (r.d_logp[-2:] == 0).all()


def test_preference_loss_gradient_against_differences(cuda_device):
    logp, ref, starts = inputs([30, 20, 0, 15, 7, 7], 3, 4, 6)
    w = torch.rand(3, device="cuda", generator=gen(1))
    for kw in (dict(beta=0.7, label_smoothing=0.1, weights=w), dict(beta=0.5, kind="ipo"), dict(beta=0.1, kind="hinge", average=True)):
        lr = logp.clone().requires_grad_()
        up = torch.rand(3, device="cuda", generator=gen(2))
        loss, rewards = A.preference_loss(lr, ref, starts, **kw)
        assert not rewards.requires_grad
        (loss * up).sum().backward()
        f = lambda x: float((formula(x, ref, starts, **kw)[0] * up).sum())  # noqa: E731
        for seed in range(3):
            d = torch.randn(logp.shape, generator=gen(seed), device="cuda", dtype=torch.float64)
            step = 1e-5
            want = (f(logp.double() + step * d) - f(logp.double() - step * d)) / (2 * step)
            size = float((lr.grad.double() * d).abs().sum())
            assert abs(float((lr.grad.double() * d).sum()) - want) <= 400 * U * size + 1e-6 * size + 1e-8


def test_preference_loss_on_another_stream_and_in_graphs(cuda_device):
    logp, ref, starts = inputs(lengths(60, 500, 9), 9)
    want = T.preference_loss(logp, ref, starts)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = T.preference_loss(logp, ref, starts)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got.loss, want.loss) and torch.equal(got.d_logp, want.d_logp)
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(T.preference_loss(logp, ref, starts))
        graphs.append(g)
    logp.mul_(0.5)
    want = T.preference_loss(logp, ref, starts)
    for g, got in zip(graphs, outs):
        g.replay()
        assert torch.equal(got.loss, want.loss) and torch.equal(got.rewards, want.rewards) and torch.equal(got.d_logp, want.d_logp)
