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


def accepted(lib, steps, a, b, c):
    """Whether a call with this polynomial gets as far as asking for its workspace, which comes after the polynomial and before the device"""
    m = matrices((300, 700), 1)
    D = C.c_double
    code = lib.ssgd_orthogonalize(m.ctypes.data, 1, S.FMT_F32, 1, steps, D(a), D(b), D(c), D(1e-7), None, 0, None)
    assert code in (S.EINVAL, S.EWORKSPACE)
    return code == S.EWORKSPACE


def reach(steps, a, b, c, points=200_001):
    """The largest that the polynomial makes of many singular values on the way, and at the end (or once it is far beyond)"""
    s, way = np.linspace(0, 1, points), 1.0
    for _ in range(steps):
        way = max(way, np.abs(s).max())
        if way > 1e6:
            break
        q = s * s
        s = s * (a + q * (b + c * q))
    return way, np.abs(s).max()


# between the points of a coarse grid on [0, 1] these leave every range
@pytest.mark.parametrize("steps,a,b,c", [(8, 2.5820751723704674, -5.537853914649217, 1.9408113825834064),
                                         (7, 2.5156164553125673, -4.720735474494571, 1.1852813270571287),
                                         (6, 3.234364782498459, -6.501583412432502, 2.1991137019973506),
                                         (5, 3.7428638927267945, -8.380319386742006, 3.4978279724879764),
                                         (5, 2.653961100954992, -4.808708104907779, 1.1347372981776571),
                                         (3, 3.5222579363973665, -8.513114138869676, 3.6355787279214278)])
def test_polynomials_that_leave_the_range_between_the_points_of_a_grid(lib, steps, a, b, c):
    assert max(reach(steps, a, b, c)) > 8
    assert not accepted(lib, steps, a, b, c)


def test_polynomials_that_stay_in_range_are_accepted(lib):
    for steps in (1, 2, 5, 10, 32):
        for poly in ((3.4445, -4.7750, 2.0315), (1.5, -0.5, 0.0), (1.875, -1.25, 0.375), (2.0, -1.5, 0.5), (1.0, 0.0, 0.0), (0.0, 0.0, 0.0), (-1.5, 0.5, 0.0)):
            assert accepted(lib, steps, *poly), (steps, poly)
    assert accepted(lib, 1, 2.0, 0.0, 0.0) and accepted(lib, 2, 2.0, 0.0, 0.0) and accepted(lib, 1, 7.9, 0.0, 0.0)
    assert not accepted(lib, 3, 2.0, 0.0, 0.0) and not accepted(lib, 2, 7.9, 0.0, 0.0) and not accepted(lib, 1, 8.1, 0.0, 0.0)
    for bad in (float("nan"), float("inf"), -float("inf"), 1e200):
        for poly in ((bad, 0.0, 0.0), (1.0, bad, 0.0), (1.0, 0.0, bad)):
            assert not accepted(lib, 1, *poly)


def test_the_range_is_that_of_a_fine_grid(lib):
    rng = np.random.default_rng(1)
    for i in range(300):
        a, b, c = rng.uniform(0, 6), rng.uniform(-12, 6), rng.uniform(-5, 6)
        if i % 2:
            a, b, c = 3.4445 * rng.uniform(0.8, 1.25), -4.775 * rng.uniform(0.8, 1.25), 2.0315 * rng.uniform(0.8, 1.25)
        steps = int(rng.integers(1, 8))
        way, end = reach(steps, a, b, c, 20_001)
        if way > 4 or end > 8:
            assert not accepted(lib, steps, a, b, c), (steps, a, b, c)
        elif way < 3.9 and end < 7.8 and 16 * abs(b) + 256 * abs(c) * (way / 4) ** 4 < 47:
            assert accepted(lib, steps, a, b, c), (steps, a, b, c)
