"""ssgd_orthogonalize through the C ABI: the field for a momentum is not used, whatever it holds."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_1903_04488_b200 import ssgd as S
from paper_1903_04488_b200 import train_ops as T

P = 1 << 12
D = C.c_double


def call(x, out, m, products=0, ws=None, bytes=0, stream=None):
    """x, out, m: addresses and the size"""
    rows, cols = x[1]
    d = np.array([[out, x[0], m, cols, cols, rows, cols, 0]], dtype=np.int64)
    return S.lib().ssgd_orthogonalize(d.ctypes.data, 1, S.FMT_F32, products, 5, D(3.4445), D(-4.775), D(2.0315), D(1e-7), ws, bytes, stream)


def test_an_address_that_is_not_used_is_not_checked():
    assert call((P, (300, 200)), P, P + 2) == S.EWORKSPACE          # as with m = 0: the workspace is looked at after the matrices
    assert call((P, (300, 200)), P, 0) == S.EWORKSPACE


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(60, 100), (300, 200)])
def test_a_momentum_that_is_given_is_neither_read_nor_written(cuda_device, shape):
    g = torch.Generator(device="cuda").manual_seed(1)
    x, m = torch.randn(*shape, generator=g, device="cuda"), torch.randn(*shape, generator=g, device="cuda")
    before, out = m.clone(), torch.empty_like(x)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    assert call((x.data_ptr(), shape), out.data_ptr(), m.data_ptr(), ws=ws.data_ptr(), bytes=ws.numel(), stream=torch.cuda.current_stream().cuda_stream) == S.OK
    assert torch.equal(out, T.orthogonalize(x)) and torch.equal(m, before)
    T.status()
