"""Calls on two streams at once, large matrices and small ones beside each other, and parameters that lie anywhere in one flat vector."""
import pytest
import torch

from paper_1903_04488_b200 import train_ops as T

from .test_gpu_orthogonalize import rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_two_streams_at_once(cuda_device, dtype):
    xs = [rand(8, 700, 900, seed=1).to(dtype), rand(300, 64, 192, seed=2).to(dtype), rand(300, 64, 64, seed=3).to(dtype), rand(3, 1100, 500, seed=4).to(dtype)]
    want = [T.orthogonalize(x) for x in xs]
    T.status()
    streams = [torch.cuda.Stream() for _ in xs]
    got = [[] for _ in xs]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        for s, x, to in zip(streams, xs, got):
            with torch.cuda.stream(s):
                to.append(T.orthogonalize(x))
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    for w, ys in zip(want, got):
        assert all(torch.equal(y, w) for y in ys)
    T.status()


@pytest.mark.parametrize("pdtype,gdtype", [(torch.float32, torch.float32), (torch.float32, torch.float16), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)])
def test_parameters_that_lie_anywhere_take_the_same_step(cuda_device, pdtype, gdtype):
    """Pieces of flat vectors at odd offsets against the same tensors by themselves: equal to the bit, and nothing beside them is touched."""
    shapes = [(64, 128), (301, 517), (33, 70), (1, 40), (700, 200), (2, 130, 260), (128, 256)]
    gap = 3
    total = sum(gap + torch.Size(s).numel() for s in shapes) + gap

    def pieces(flat):
        out, at = [], 0
        for s in shapes:
            n = torch.Size(s).numel()
            out.append(flat[at + gap: at + gap + n].view(s))
            at += gap + n
        return out

    p, g, m = rand(total, seed=1).to(pdtype), rand(total, seed=2).to(gdtype), rand(total, seed=3)
    before = p.clone(), g.clone(), m.clone()
    apart = [[t.clone() for t in pieces(f)] for f in (p, g, m)]
    a = T.Muon(pieces(p), m=pieces(m), weight_decay=0.1)
    b = T.Muon(apart[0], m=apart[2], weight_decay=0.1)
    for _ in range(2):
        a.step(pieces(g))
        b.step(apart[1])
    T.status()
    for mine, other in ((p, apart[0]), (m, apart[2])):
        assert all(torch.equal(x, y) for x, y in zip(pieces(mine), other))
    assert torch.equal(g, before[1])
    for now, then in ((p, before[0]), (m, before[2])):
        for t in pieces(now) + pieces(then):
            t.zero_()
        assert torch.equal(now, then)
