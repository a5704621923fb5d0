"""Matrices that one CTA takes, in calls that follow one another closely."""
import pytest
import torch

from paper_1903_04488_b200 import train_ops as T

from .test_gpu_orthogonalize import check, rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_launches_that_need_unlike_tensor_memory_follow_one_another(cuda_device, dtype):
    """64 columns of tensor memory, then 256, then 128, each on every SM several times over: the second may start while the first runs, and two of
    its CTAs and one of the first's fit an SM's shared memory, but not its tensor memory."""
    shapes = [(64, 64), (64, 192), (64, 128), (192, 64), (60, 50)]
    xs = [rand(600, *s, seed=i).to(dtype) for i, s in enumerate(shapes)]
    alone = []
    for x in xs:
        alone.append(T.orthogonalize(x))
        T.status()
    for _ in range(20):
        together = [T.orthogonalize(x) for x in xs]
    T.status()
    for x, a, b in zip(xs, alone, together):
        assert torch.equal(a, b)
        check(x[:5], b[:5], 1 if dtype == torch.bfloat16 else 3)
