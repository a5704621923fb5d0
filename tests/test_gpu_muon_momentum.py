"""The weight of the gradient in the momentum is 1 - momentum as the caller gave it, not of a momentum rounded to fp32."""
import pytest
import torch

from paper_1903_04488_b200 import train_ops as T

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("momentum", [0.0, 0.9, 0.95, 0.999, 0.9999, 0.99999])
@pytest.mark.parametrize("gdtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(64, 128), (300, 517)])
def test_the_first_momentum_is_the_gradients_share(cuda_device, shape, gdtype, momentum):
    """From zeros m = (1 - momentum) g: the rounding of the factor and that of the product, half a unit each.  The next one is (1 + momentum) g of that:
    those two once more (1 + momentum <= 2 times), the rounding of momentum (1) and that of the sum (2): 7 half units of the first at most."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    p = torch.randn(*shape, generator=gen, device="cuda")
    g = torch.randn(*shape, generator=gen, device="cuda").to(gdtype)
    opt = T.Muon([p], momentum=momentum)
    opt.step([g])
    first = (1 - momentum) * g.double()
    assert ((opt.m[0].double() - first).abs() <= 2.01 * U * first.abs()).all()
    opt.step([g])
    second = (1 + momentum) * first
    assert ((opt.m[0].double() - second).abs() <= 7.01 * U * first.abs()).all()
    T.status()
