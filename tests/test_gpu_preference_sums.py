"""What the preference loss' sums hold: masks of the lowest number, several to a sequence, and differences of more than 24 bits.

The inputs are such that every sum is exact in 64 bits; what remains is the rounding of x and of the rewards to fp32 (U = 2^-24), two of 64 bits
before it, and the loss and its slope, a few fp32 operations: 16 U."""
import math

import numpy as np
import pytest
import torch

from paper_1903_04488_b200 import train_ops as T

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
LOWEST = torch.finfo(torch.float32).min
# lengths of the sequences: in one CTA, over several CTAs, sequences beyond what a CTA keeps in a table, short and long ones among them
LENS = [[50, 50] * 6, [3000, 2500] * 8, [20000, 30001] * 3, [5, 7] * 300, ([3] * 90 + [200, 150]) * 40]


def expected(logp, ref, at, beta):
    """D per sequence, loss and slope per pair, in 64 bits"""
    diff = logp.double() if ref is None else logp.double() - ref.double()
    D = np.array([math.fsum(diff[a:b].tolist()) for a, b in zip(at, at[1:])]).reshape(-1, 2)
    x = float(np.float32(beta)) * (D[:, 0] - D[:, 1])
    soft = np.log1p(np.exp(-np.abs(x)))
    lose = np.where(x >= 0, np.exp(-np.abs(x)), 1.0) / (1 + np.exp(-np.abs(x)))
    return D, x, np.maximum(-x, 0) + soft, -lose * float(np.float32(beta))


def check(logp, ref, at, beta, r):
    D, x, loss, slope = expected(logp.cpu(), None if ref is None else ref.cpu(), at, beta)
    got = [t.cpu().double().numpy() for t in (r.loss, r.rewards, r.d_logp)]
    rewards = float(np.float32(beta)) * D.T
    assert (np.abs(got[1] - rewards) <= 2 * U * np.abs(rewards)).all()
    off = 2 * U * np.abs(x)                          # of x; the loss has slope 1 at most, its slope 1/4
    assert (np.abs(got[0] - loss) <= off + 16 * U * (loss + 1)).all()
    tol = beta * (np.minimum(off, 4) / 4 + 16 * U)
    for p in range(len(x)):
        a, b, c = at[2 * p: 2 * p + 3]
        assert (np.abs(got[2][a:b] - slope[p]) <= tol[p]).all() and (np.abs(got[2][b:c] + slope[p]) <= tol[p]).all()


@pytest.mark.parametrize("lens", LENS, ids=lambda v: "%dx%d" % (len(v), v[0]))
@pytest.mark.parametrize("before", [0, 8100])
def test_masks_of_the_lowest_number_several_to_a_sequence(cuda_device, lens, before):
    """Their sum is beyond fp32, and what the loss needs of it is not: the same number of masks in both sequences leaves x = 0."""
    at = (before + np.concatenate([[0], np.cumsum(lens)])).tolist()
    g = torch.Generator(device="cuda").manual_seed(len(lens))
    logp = -torch.rand(at[-1] + 5, generator=g, device="cuda")
    masks = []
    for s, (a, b) in enumerate(zip(at, at[1:])):
        if s % 6 < 4:                                # pairs: as many in both, more in the second, none
            n = (2, 2, 2, 3)[s % 6]
            masks += [a, b - 1, (a + b) // 2][:n]
    logp[torch.tensor(masks, device="cuda")] = LOWEST
    starts = torch.tensor(at, device="cuda")
    for ref in (None, torch.zeros_like(logp)):
        r = T.preference_loss(logp, ref, starts)
        assert all(t.isfinite().all() for t in (r.loss, r.rewards, r.d_logp))
        check(logp, ref, at, 0.1, r)
    # masked in the reference too: nothing is left of them
    both = T.preference_loss(logp, torch.where(logp == LOWEST, logp, 0.0), starts)
    clean = T.preference_loss(torch.where(logp == LOWEST, 0.0, logp), None, starts)
    assert (both.rewards.double() - clean.rewards.double()).abs().max() <= 4 * U * clean.rewards.abs().max()
    # and what is not finite stays so
    logp[at[0]] = -math.inf
    r = T.preference_loss(logp, None, starts)
    assert r.rewards[0, 0] == -math.inf and r.loss[0] == math.inf and r.loss[1:].isfinite().all()


@pytest.mark.parametrize("lens", [[100, 100], [1 << 17, 1 << 17], [10] * 400, ([3] * 90 + [200, 200]) * 40, [4097, 4097] * 6],
                         ids=lambda v: "%dx%d" % (len(v), v[0]))
@pytest.mark.parametrize("before", [0, 1])
def test_differences_keep_the_bits_that_one_number_does_not(cuda_device, lens, before):
    """logp - ref_logp = -1 - 2^-26 in the first sequence of each pair and -1 in the second: rounded to fp32 they are the same, and the loss log 2."""
    at = (before + np.concatenate([[0], np.cumsum(lens)])).tolist()
    logp = torch.full((at[-1],), -1.0, device="cuda")
    ref = torch.zeros_like(logp)
    for a, b in zip(at[::2], at[1::2]):
        ref[a:b] = 2.0 ** -26
    beta = 2.0 ** 26 / max(lens)                     # x = -1 for the longest
    r = T.preference_loss(logp, ref, torch.tensor(at, device="cuda"), beta=beta)
    check(logp, ref, at, beta, r)
