"""Orthogonalised matrices and the Muon step against the iteration in 64 bits.

Errors are norms of differences over norms of results.  With three products the result is held to what the same iteration in fp32
(torch, on the same input) is off by, twice that, plus 2^-19: a sum of two fp16 numbers keeps 22 bits, five steps of three products.
With one product every operand is off by up to 2^-12 of each element, 2^-12 / sqrt 3 on average; near the singular value 1 a step passes on
(2 |b| + 4 |c|) = 18 of that from A and B's operands, 2.5e-3, the steps before the last less than half as much together, independently: 4e-3.
An output in 16 bits adds its own half unit."""
import copy
import math

import pytest
import torch

from paper_1903_04488_b200 import train_ops as T

pytestmark = pytest.mark.gpu

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
ONE_PRODUCT = 4e-3
C = T.QUINTIC


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rand(*shape, seed=0):
    return torch.randn(*shape, generator=gen(seed), device="cuda")


def iterate(x, steps=5, coefficients=C, eps=1e-7):
    a, b, c = coefficients
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + eps)
    tall = x.shape[-2] > x.shape[-1]
    x = x.mT if tall else x
    for _ in range(steps):
        g = x @ x.mT
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.mT if tall else x


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


def check(x, y, products, **kw):
    want = iterate(x.double(), **kw)
    allowed = 2 * off(iterate(x.float(), **kw), want) + 2.0 ** -19 if products == 3 else ONE_PRODUCT
    assert off(y, want) <= allowed + HALF[y.dtype], (tuple(x.shape), x.dtype, products)


SIZES = [(1, 1), (1, 9), (9, 1), (2, 3), (31, 33), (64, 64), (64, 128), (128, 64), (65, 65), (128, 128), (129, 127), (100, 700), (700, 100), (256, 256),
         (257, 300), (320, 1000), (1000, 320), (513, 513), (640, 1280), (1100, 900)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_orthogonalize(cuda_device, rows, cols, dtype):
    x = rand(rows, cols, seed=rows).to(dtype)
    for products in (None, 1, 3):
        y = T.orthogonalize(x, products=products)
        assert y.dtype == dtype and y.shape == x.shape
        check(x, y, products or (1 if dtype == torch.bfloat16 else 3))
    T.status()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_orthogonalize_of_unlike_singular_values(cuda_device, dtype):
    """A few strong directions over noise, a steep fall, all but one direction: what is far below the largest is not lost."""
    m, n = 200, 300
    u, v = torch.linalg.qr(rand(m, m, seed=1).double())[0], torch.linalg.qr(rand(n, n, seed=2).double())[0]
    for s in (torch.cat([torch.full((8,), 1.0), torch.full((m - 8,), 0.02)]), torch.logspace(0, -4, m), torch.cat([torch.ones(1), torch.full((m - 1,), 1e-3)])):
        x = (u * s.to(u) @ v[:m]).to(dtype)
        for products in (1, 3):
            check(x, T.orthogonalize(x.float(), products=products), products)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_orthogonalize_of_strided_batches_and_in_place(cuda_device, dtype):
    x = rand(3, 100, 150, seed=3).to(dtype)
    each = torch.stack([T.orthogonalize(m) for m in x])
    assert torch.equal(T.orthogonalize(x), each)
    wide = rand(100, 400, seed=4).to(dtype)
    for cut in (slice(0, 150), slice(8, 158), slice(3, 153)):
        piece = wide[:, cut]
        want = T.orthogonalize(piece.contiguous())
        assert torch.equal(T.orthogonalize(piece), want)
        host = wide.clone()
        out = T.orthogonalize(host[:, cut], out=host[:, cut])
        assert torch.equal(out, want) and torch.equal(host[:, cut.stop:], wide[:, cut.stop:]) and torch.equal(host[:, : cut.start], wide[:, : cut.start])


def test_orthogonalize_of_zeros_magnitudes_and_values_that_are_not_finite(cuda_device):
    x = torch.zeros(5, 70, 90, device="cuda")
    x[1:] = rand(4, 70, 90, seed=5)
    x[2] *= 1e30                               # its squares are beyond fp32
    x[3] *= 1e-3
    x[4, 3, 4] = math.nan
    y = T.orthogonalize(x)
    assert (y[0] == 0).all() and y[4].isnan().all()
    for i in (1, 2, 3):
        check(x[i], y[i], 3)
    tiny = rand(70, 90, seed=5) * 1e-30        # far below eps: near zero, which is zero
    assert T.orthogonalize(tiny).abs().max() < 1e-10
    exact = T.orthogonalize(tiny, eps=0.0)
    assert off(exact, iterate(rand(70, 90, seed=5).double(), eps=0.0)) < 1e-5
    for big in (3e36, 5e37):                   # the norm itself is beyond fp32
        for shape in ((70, 90), (300, 200)):
            y = rand(*shape, seed=6).clamp(-6, 6)
            assert off(T.orthogonalize(y * big), iterate((y * big).double())) < 1e-5
            assert off(T.orthogonalize((y * big).bfloat16()), iterate((y * big).bfloat16().double())) < ONE_PRODUCT + 2.0 ** -8
    x[1, 0, 0] = math.inf
    assert T.orthogonalize(x[1]).isnan().any() and T.orthogonalize(torch.zeros(3, 3, device="cuda"), eps=0.0).isnan().all()


@pytest.mark.parametrize("steps,coefficients", [(1, C), (2, C), (7, C), (6, (1.5, -0.5, 0.0)), (3, (1.875, -1.25, 0.375)), (4, (2.0, 0.0, 0.0))])
def test_orthogonalize_with_other_polynomials(cuda_device, steps, coefficients):
    for shape in ((150, 90), (90, 300)):
        x = rand(*shape, seed=steps)
        if coefficients == (2.0, 0.0, 0.0):
            x = x * 0 + torch.eye(*shape, device="cuda")      # exactly 16 x / |x|: powers of two
            steps = 1
        check(x, T.orthogonalize(x, steps=steps, coefficients=coefficients), 3, steps=steps, coefficients=coefficients)


def test_orthogonalize_repeats_bit_for_bit_on_streams_and_in_graphs(cuda_device):
    x = rand(6, 200, 333, seed=7).bfloat16()
    want = T.orthogonalize(x)
    assert torch.equal(T.orthogonalize(x), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = T.orthogonalize(x)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(T.orthogonalize(x))
        graphs.append(g)
    x.copy_(rand(6, 200, 333, seed=8))
    want = T.orthogonalize(x)
    for g, got in zip(graphs, outs):
        g.replay()
    assert all(torch.equal(got, want) for got in outs)
    T.status()


def test_orthogonalize_of_many_matrices_in_groups(cuda_device):
    x = rand(500, 40, 24, seed=9).half()
    y = T.orthogonalize(x)
    assert torch.equal(y[:3], T.orthogonalize(x[:3])) and torch.equal(y[-3:], T.orthogonalize(x[-3:]))
    check(x, y, 3)


# ---- the optimizer -----------------------------------------------------------------------------------


def plain_step(p, g, m, lr, momentum, nesterov, decay, scale, grad_scale=1.0):
    p, g, m = p.double(), g.double() * grad_scale, m.double()
    m = momentum * m + (1 - momentum) * g
    u = momentum * m + (1 - momentum) * g if nesterov else m
    return p * (1 - lr * decay) - lr * scale * iterate(u), m


SHAPES = [(64, 128), (128, 64), (33, 70), (5, 200, 100), (300, 300), (1, 40)]


@pytest.mark.parametrize("pdtype,gdtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.bfloat16),
                                           (torch.bfloat16, torch.float32), (torch.float32, torch.float16)])
@pytest.mark.parametrize("nesterov,scale", [(True, "spectral"), (False, "rms"), (True, 0.3)])
def test_muon_step(cuda_device, pdtype, gdtype, nesterov, scale):
    params = [(0.1 * rand(*s, seed=i)).to(pdtype) for i, s in enumerate(SHAPES)]
    grads = [rand(*s, seed=50 + i).to(gdtype) for i, s in enumerate(SHAPES)]
    start = [rand(*s, seed=90 + i) for i, s in enumerate(SHAPES)]
    opt = T.Muon(params, lr=0.02, momentum=0.9, nesterov=nesterov, weight_decay=0.1, scale=scale, m=[m.clone() for m in start])
    before = [p.clone() for p in params]
    share = torch.full((1,), 0.5, device="cuda")
    grads[2] = None                            # left alone
    opt.step(grads, grad_scale=share)
    for i, s in enumerate(SHAPES):
        if grads[i] is None:
            assert torch.equal(params[i], before[i]) and torch.equal(opt.m[i], start[i])
            continue
        factor = {"spectral": max(1.0, s[-2] / s[-1]) ** 0.5, "rms": 0.2 * max(s[-2:]) ** 0.5}.get(scale, scale)
        p, m = plain_step(before[i], grads[i], start[i], 0.02, 0.9, nesterov, 0.1, factor, 0.5)
        assert ((opt.m[i].double() - m).abs() <= 4 * 2.0 ** -24 * (start[i].double().abs() + grads[i].double().abs())).all()
        update = (p - before[i].double() * (1 - 0.02 * 0.1)).norm()
        allowed = float(update) * (ONE_PRODUCT if pdtype == torch.bfloat16 else 2e-5) + float((before[i].double().abs() + p.abs()).norm()) * HALF[pdtype]
        assert float((params[i].double() - p).norm()) <= allowed
    T.status()


def test_muon_follows_its_parameters_and_is_copied(cuda_device):
    params = [rand(40, 60, seed=i).requires_grad_() for i in range(3)]
    with torch.no_grad():
        opt = T.Muon(params)
        version = params[0]._version
        grads = [rand(40, 60, seed=9 + i) for i in range(3)]
        opt.step(grads)
        assert params[0]._version > version
        twin = copy.deepcopy(opt)
        opt.step(grads)
        twin.step(tuple(grads))
        assert all(torch.equal(a, b) for a, b in zip(opt.params, twin.params)) and opt.params[0].data_ptr() != twin.params[0].data_ptr()
        opt.step([None] * 3)
        assert all(torch.equal(a, b) for a, b in zip(opt.params, twin.params))
        params[0].data = rand(40, 60, seed=77)                 # other storage
        opt.step(grads)
        assert not torch.equal(params[0], rand(40, 60, seed=77))


def test_muon_in_a_graph_touches_nothing_else(cuda_device):
    flat = rand(3 * 2000 + 14, seed=3)
    params = [flat[2000 * i + 7 * (i > 0): 2000 * i + 7 * (i > 0) + 2000].view(40, 50) for i in range(3)]
    before = flat.clone()
    opt = T.Muon(params, lr=0.1)
    grads = [rand(40, 50, seed=i) for i in range(3)]
    twin = T.Muon([p.clone() for p in params], lr=0.1)
    twin.step(grads)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        opt.step(grads)
    assert torch.equal(flat, before)
    g.replay()
    assert all(torch.equal(a, b) for a, b in zip(params, twin.params))
    assert torch.equal(flat[2000:2007], before[2000:2007]) and torch.equal(flat[-7:], before[-7:])


def test_muon_refuses_what_does_not_fit(cuda_device):
    p = [rand(8, 9), rand(8, 9)]
    for bad in (lambda: T.Muon([rand(8)]), lambda: T.Muon([rand(8, 9).half()]), lambda: T.Muon([rand(9, 8).t()]), lambda: T.Muon(p, m=[rand(8, 9).half(), rand(8, 9)])):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: T.Muon([]), lambda: T.Muon([p[0], p[0]]), lambda: T.Muon(p, scale="none"), lambda: T.Muon(p, m=[rand(8, 9)])):
        with pytest.raises(ValueError):
            bad()
    opt = T.Muon(p)
    before = [t.clone() for t in p]
    for grads in ([rand(8, 9)], [rand(8, 9), rand(9, 8)], [rand(8, 9), rand(8, 9).half()], [rand(8, 9), rand(8, 18)[:, ::2]], [rand(8, 9).cpu(), rand(8, 9)]):
        with pytest.raises((TypeError, ValueError)):
            opt.step(grads)
    with pytest.raises(T.S.SsgdError):
        opt.step([rand(8, 9)] * 2, lr=-1.0)
    with pytest.raises(T.S.SsgdError):
        T.orthogonalize(p[0], coefficients=(9.0, 9.0, 9.0))
    with pytest.raises(T.S.SsgdError):
        T.orthogonalize(p[0], steps=0)
    with pytest.raises(TypeError):
        T.orthogonalize(rand(8))
    assert all(torch.equal(a, b) for a, b in zip(p, before))
