"""The scale of Muon's updates and the way the weights are stored: [out][in] for "spectral", [in][out] for "spectral_t"."""
import pytest
import torch

from paper_1903_04488_b200 import train_lm, train_ops as T

pytestmark = pytest.mark.gpu


def rand(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


@pytest.mark.parametrize("shape", [(64, 128), (128, 64), (3, 40, 100), (300, 1200), (50, 50)])
def test_a_matrix_and_its_transpose_take_the_same_step(cuda_device, shape):
    """W and W' stored the other way round: the updates are each other's transposes to the iteration's own 2e-5 (three products, as in the tests
    of the matrices); a scale for the other orientation would be off by the square root of the sides' ratio."""
    p, g = rand(*shape), rand(*shape, seed=1)
    a, b = p.clone(), p.mT.contiguous()
    T.Muon([a], scale="spectral").step([g])
    T.Muon([b], scale="spectral_t").step([g.mT.contiguous()])
    off = float((a - b.mT).double().norm()), float((a - p).double().norm())
    assert off[0] <= 2 * (2e-5 * off[1] + 2.0 ** -24 * float(p.double().norm()))
    rows, cols = shape[-2:]
    assert T.Muon([p], scale="spectral").scales == [max(1.0, rows / cols) ** 0.5]
    assert T.Muon([p], scale="spectral_t").scales == [max(1.0, cols / rows) ** 0.5]


def test_tuning_scales_by_outputs_over_inputs(cuda_device, monkeypatch):
    seen = []

    class Spy(train_lm.Tuner):
        def __init__(self, *a, **k):
            super().__init__(*a, **k)
            seen.append(self)

    monkeypatch.setattr(train_lm, "Tuner", Spy)
    model = train_lm.Model(64, 32, 2, cuda_device)
    train_lm.tune(model, torch.randperm(64, device="cuda"), torch.Generator(device="cuda").manual_seed(1), 1, 64, quiet=True)
    # x @ W: rows are inputs, columns outputs; 32 -> 64 widens, 64 -> 32 narrows
    assert [tuple(p.shape) for p in seen[0].blocks] == [(32, 64), (64, 32)] * 2
    assert seen[0].muon.scales == [2.0 ** 0.5, 1.0] * 2
