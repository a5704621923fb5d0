"""Orthogonalised matrices that one launch cannot hold: tiles of 256 columns, more tiles than pairs of CTAs, several sets of launches
in one workspace, unlike matrices together.

The tiles of a product have 256 columns where that is less work for the busiest pair of CTAs (148 SMs, 74 pairs): by that rule so
have all three products of MANY, those of half of the matrices in UNLIKE, and of the rest those whose tiles are few have 128.  Tolerances as
for the small ones: they count roundings of operands, which the size does not change."""
import pytest
import torch

from paper_1903_04488_b200 import train_ops as T

from .test_gpu_orthogonalize import HALF, ONE_PRODUCT, check, plain_step, rand

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
# batch, rows, cols: ragged in both directions, both orientations, a single large one
MANY = [(8, 1003, 1101), (8, 1100, 1000), (20, 500, 700), (1, 2900, 3001), (1, 3000, 2900)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,rows,cols", MANY)
def test_wide_tiles_and_more_of_them_than_pairs(cuda_device, batch, rows, cols, dtype):
    x = rand(batch, rows, cols, seed=rows).to(dtype)
    for products in (1, 3):
        y = T.orthogonalize(x, products=products)
        for a, b in zip(x, y):
            check(a, b, products)
        # in the same order, whoever is first
        assert torch.equal(T.orthogonalize(x, products=products), y)
    T.status()


@pytest.mark.parametrize("dtype", TYPES)
def test_groups_of_large_matrices_share_the_workspace(cuda_device, dtype):
    """More matrices than one set of launches takes: the second set writes where the first one's tiles have just been read."""
    x = rand(500, 260, 70, seed=9).to(dtype)
    y = T.orthogonalize(x)
    check(x[::37], y[::37], 1 if dtype == torch.bfloat16 else 3)
    for cut in (slice(0, 224), slice(224, 448), slice(448, 500)):
        assert torch.equal(T.orthogonalize(x[cut]), y[cut])
    T.status()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(600, 801), (801, 600)])
def test_large_matrices_in_place_and_in_rows_that_are_not_adjacent(cuda_device, rows, cols, dtype):
    wide = rand(rows, cols + 99, seed=4).to(dtype)
    for at in (0, 8, 3):
        cut = slice(at, at + cols)
        want = T.orthogonalize(wide[:, cut].contiguous())
        assert torch.equal(T.orthogonalize(wide[:, cut]), want)
        host = wide.clone()
        out = T.orthogonalize(host[:, cut], out=host[:, cut])
        assert torch.equal(out, want)
        assert torch.equal(host[:, : at], wide[:, : at]) and torch.equal(host[:, cut.stop:], wide[:, cut.stop:])


UNLIKE = [(300, 517), (517, 300), (2000, 2001), (64, 128), (1700, 2500), (3, 700, 260), (70, 5001), (40, 24), (5001, 70)]


@pytest.mark.parametrize("pdtype,gdtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.bfloat16)])
def test_a_step_over_unlike_matrices(cuda_device, pdtype, gdtype):
    params = [(0.1 * rand(*s, seed=i)).to(pdtype) for i, s in enumerate(UNLIKE)]
    grads = [rand(*s, seed=50 + i).to(gdtype) for i, s in enumerate(UNLIKE)]
    before = [p.clone() for p in params]
    opt = T.Muon(params, lr=0.02, momentum=0.9, weight_decay=0.1, scale=0.5)
    for step in range(2):
        moved = [p.clone() for p in params], [m.clone() for m in opt.m]
        opt.step(grads)
        for i in range(len(UNLIKE)):
            p, m = plain_step(moved[0][i], grads[i], moved[1][i], 0.02, 0.9, True, 0.1, 0.5)
            assert ((opt.m[i].double() - m).abs() <= 4 * 2.0 ** -24 * (moved[1][i].double().abs() + grads[i].double().abs())).all(), i
            update = (p - moved[0][i].double() * (1 - 0.02 * 0.1)).norm()
            allowed = float(update) * (ONE_PRODUCT if pdtype == torch.bfloat16 else 2e-5) + float((moved[0][i].double().abs() + p.abs()).norm()) * HALF[pdtype]
            assert float((params[i].double() - p).norm()) <= allowed, i
    # alone they come to the same but for the width of the tiles they are given
    twin = [before[0].clone(), before[3].clone()]
    other = T.Muon(twin, lr=0.02, momentum=0.9, weight_decay=0.1, scale=0.5)
    for _ in range(2):
        other.step([grads[0], grads[3]])
    assert torch.equal(twin[1], params[3])
    assert float((twin[0].double() - params[0].double()).norm()) <= 2 * (ONE_PRODUCT if pdtype == torch.bfloat16 else 2e-5) * float((params[0] - before[0]).double().norm()) + 2 * HALF[pdtype] * float(params[0].double().norm())
    T.status()


def test_a_large_call_in_a_graph_repeats_itself(cuda_device):
    x = rand(8, 1003, 1101, seed=7).bfloat16()
    many = rand(230, 260, 70, seed=8)
    want = T.orthogonalize(x), T.orthogonalize(many)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = T.orthogonalize(x), T.orthogonalize(many)
        graphs.append((g, out))
    for _ in range(3):
        for g, out in graphs:
            g.replay()
    for _, out in graphs:
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    T.status()
