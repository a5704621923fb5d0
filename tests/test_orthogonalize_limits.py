"""The workspace of orthogonalised matrices and the polynomials that are refused: host side only, no GPU is needed."""
import ctypes as C

import numpy as np
import pytest

from paper_1903_04488_b200 import build as B
from paper_1903_04488_b200 import ssgd as S

P = 1 << 12


@pytest.fixture(scope="module")
def lib():
    B.build()
    return S.lib()


def matrices(shape, count):
    """ssgd_matrix: out, in, m, ld_out, ld_in, rows, cols, scale"""
    out = np.zeros((count, 8), dtype=np.int64)
    out[:, :7] = [P, P, P, shape[1], shape[1], shape[0], shape[1]]
    return out


def workspace(lib, shape, count, products=1):
    need = S._sz()
    m = matrices(shape, count)
    assert lib.ssgd_orthogonalize_workspace(m.ctypes.data, count, S.FMT_F32, products, C.byref(need)) == S.OK
    return need.value


def up(n):
    return (n + 63) // 64 * 64


@pytest.mark.parametrize("shape", [(1, 1 << 20), (1 << 20, 1), (8, 4096), (3, 5000), (64, 70000), (65, 300), (1000, 2800)])
@pytest.mark.parametrize("products", [1, 3])
def test_the_workspace_counts_sides_rounded_up_and_stops_growing(lib, shape, products):
    rows, cols = up(shape[0]), up(shape[1])
    lo = min(rows, cols)
    each = 8 * rows * cols + (4 if products == 1 else 8) * lo * lo
    one = workspace(lib, shape, 1, products)
    # d and e, a sum to a strip, which is a block of 64 x 64 at least, descriptors
    assert each <= one <= each + 8 * lo + 8 * (rows // 64) * (cols // 64) + (1 << 16)
    group = min(224, max(1, (1 << 27) // (rows * cols)))
    full = workspace(lib, shape, group, products)
    assert group * each <= full <= group * one
    for more in (group + 1, 3 * group, 1000):
        assert workspace(lib, shape, more, products) == full
    assert 8 * group * rows * cols <= 8 << 27 or group == 1
