"""What the operators of the training step refuse, before anything is launched: no GPU is needed (addresses that are
only compared, never read)."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_1903_04488_b200 import build as B
from paper_1903_04488_b200 import ssgd as S
from paper_1903_04488_b200 import train_ops as T

P = 1 << 12                                    # an aligned address


@pytest.fixture(scope="module")
def lib():
    B.build()
    return S.lib()


def call(fn, good, **bad):
    kw = dict(good)
    kw.update(bad)
    return fn(*kw.values())


def test_layer_norm_refuses(lib):
    good = dict(x=P, ld_x=64, fmt=S.FMT_BF16, w=P, b=P, fmt_w=S.FMT_F32, rows=4, n=64, eps=C.c_float(1e-5), y=P, ld_y=64, stats=P,
                stream=None)
    f = lib.ssgd_layer_norm
    for bad in (dict(rows=-1), dict(n=0), dict(n=(1 << 24) + 1, ld_x=1 << 25, ld_y=1 << 25), dict(ld_x=63), dict(ld_y=63), dict(fmt=7),
                dict(fmt=S.FMT_E4M3), dict(fmt_w=S.FMT_F16), dict(eps=C.c_float(-1.0)), dict(eps=C.c_float(float("nan"))), dict(x=None),
                dict(y=None), dict(stats=None)):
        assert call(f, good, **bad) == S.EINVAL, bad
    for bad in (dict(x=P + 1), dict(y=P + 1), dict(w=P + 2), dict(b=P + 2), dict(stats=P + 2)):
        assert call(f, good, **bad) == S.EALIGN, bad
    assert call(f, good, rows=0, x=None, y=None, stats=None) == S.OK


def test_layer_norm_backward_refuses(lib):
    need = S._sz()
    assert lib.ssgd_layer_norm_backward_workspace(4, 64, C.byref(need)) == S.OK and need.value >= 4 * 2 * 64 * 4
    small = need.value
    assert lib.ssgd_layer_norm_backward_workspace(100, 64, C.byref(need)) == S.OK and need.value > small
    for a in ((-1, 64), (4, 0), (4, (1 << 24) + 1)):
        assert lib.ssgd_layer_norm_backward_workspace(*a, C.byref(need)) == S.EINVAL
    assert lib.ssgd_layer_norm_backward_workspace(4, 64, None) == S.EINVAL
    good = dict(dy=P, ld_dy=64, x=P, ld_x=64, fmt=S.FMT_F32, w=P, fmt_w=S.FMT_F32, stats=P, rows=4, n=64, dx=P, ld_dx=64, dw=P, db=P,
                acc=0, ws=P, bytes=small, stream=None)
    f = lib.ssgd_layer_norm_backward
    for bad in (dict(dy=None), dict(x=None), dict(stats=None), dict(dx=None), dict(ld_dy=63), dict(ld_x=1), dict(ld_dx=0), dict(n=-5),
                dict(fmt_w=S.FMT_BF16), dict(fmt=3), dict(rows=-2)):
        assert call(f, good, **bad) == S.EINVAL, bad
    for bad in (dict(dy=P + 2), dict(x=P + 2), dict(dx=P + 1), dict(dw=P + 2), dict(db=P + 1), dict(ws=P + 8), dict(stats=P + 1)):
        assert call(f, good, **bad) == S.EALIGN, bad
    for bad in (dict(ws=None), dict(bytes=small - 1)):
        assert call(f, good, **bad) == S.EWORKSPACE, bad


def test_token_logprobs_refuse(lib):
    good = dict(z=P, ld=100, fmt=S.FMT_F16, ids=P, id_bytes=8, rows=3, vocab=100, scale=C.c_float(1), top=5, stats=P, idx=P, lp=P,
                stream=None)
    f = lib.ssgd_token_logprobs
    inf, nan = float("inf"), float("nan")
    for bad in (dict(z=None), dict(ids=None), dict(stats=None), dict(idx=None), dict(lp=None), dict(ld=99), dict(vocab=0), dict(rows=-1),
                dict(id_bytes=2), dict(top=-1), dict(vocab=4, top=5), dict(fmt=3), dict(scale=C.c_float(0)), dict(scale=C.c_float(-1)),
                dict(scale=C.c_float(inf)), dict(scale=C.c_float(nan)), dict(vocab=(1 << 30) + 1, ld=1 << 31)):
        assert call(f, good, **bad) == S.EINVAL, bad
    assert call(f, good, top=S.MAX_TOP + 1) == S.ETOOBIG
    for bad in (dict(z=P + 1), dict(ids=P + 4), dict(stats=P + 2), dict(idx=P + 1), dict(lp=P + 2)):
        assert call(f, good, **bad) == S.EALIGN, bad
    assert call(f, good, rows=0, z=None) == S.OK
    good = dict(z=P, ld=100, fmt=S.FMT_F32, ids=P, id_bytes=4, rows=3, vocab=100, scale=C.c_float(1), lse=P, h=P, d=P, dh=P, top=2,
                idx=P, dt=P, out=P, ld_out=100, stream=None)
    f = lib.ssgd_token_logprobs_backward
    for bad in (dict(z=None), dict(ids=None), dict(lse=None), dict(h=None), dict(idx=None), dict(dt=None), dict(out=None), dict(ld_out=99),
                dict(ld=1), dict(id_bytes=1), dict(vocab=1)):
        assert call(f, good, **bad) == S.EINVAL, bad
    for bad in (dict(z=P + 2), dict(ids=P + 1), dict(out=P + 2), dict(lse=P + 1), dict(h=P + 1), dict(d=P + 1), dict(dh=P + 1),
                dict(idx=P + 2), dict(dt=P + 2)):
        assert call(f, good, **bad) == S.EALIGN, bad
    assert call(f, good, top=33) == S.ETOOBIG


def test_adamw_refuses(lib):
    def desc(**bad):
        row = dict(p=P, g=P, m=P, v=P, ms=P, vs=P, copy=0, n=10)
        row.update(bad)
        return np.array([list(row.values())], dtype=np.int64)

    good = dict(count=1, fp=S.FMT_F32, fg=S.FMT_BF16, fs=S.FMT_E4M3, fc=S.FMT_BF16, lr=C.c_double(1e-3), b1=C.c_double(0.9),
                b2=C.c_double(0.99), eps=C.c_double(1e-8), wd=C.c_double(0.0), step=1, gs=None, sr=0, seed=0, stream=None)

    def go(row=None, **bad):
        d = desc(**(row or {}))
        return call(lambda *a: lib.ssgd_adamw_step(d.ctypes.data, *a), good, **bad)

    nan = C.c_double(float("nan"))
    for bad in (dict(count=-1), dict(fp=S.FMT_F16), dict(fp=S.FMT_E4M3), dict(fg=S.FMT_E4M3), dict(fs=S.FMT_BF16), dict(fc=S.FMT_F32),
                dict(lr=C.c_double(-1)), dict(lr=nan), dict(b1=C.c_double(1.0)), dict(b2=C.c_double(-0.1)), dict(b2=nan), dict(eps=nan),
                dict(wd=C.c_double(-1)), dict(step=0)):
        assert go(**bad) == S.EINVAL, bad
    for row in (dict(p=0), dict(g=0), dict(m=0), dict(v=0), dict(ms=0), dict(vs=0), dict(n=-1)):
        assert go(row) == S.EINVAL, row
    assert go(dict(copy=P), fp=S.FMT_BF16) == S.EINVAL
    for row in (dict(p=P + 2), dict(g=P + 1), dict(ms=P + 1), dict(vs=P + 2), dict(copy=P + 1)):
        assert go(row) == S.EALIGN, row
    assert go(dict(m=P + 2), fs=S.FMT_F32) == S.EALIGN
    assert go(gs=P + 1) == S.EALIGN
    assert lib.ssgd_adamw_step(None, *good.values()) == S.EINVAL
    assert go(dict(n=0, p=0, g=0)) == S.OK and go(count=0) == S.OK       # nothing to do: nothing is launched


def test_python_checks_name_the_argument():
    x = torch.zeros(4, 8)
    for f, name in ((lambda: T.layer_norm(x), "x"), (lambda: T.token_logprobs(x, torch.zeros(4, dtype=torch.int64)), "logits"),
                    (lambda: T.layer_norm_backward(x, x, None, x), "x"), (lambda: T.AdamW([x]), "params")):
        with pytest.raises(TypeError, match=name):
            f()
    with pytest.raises(ValueError, match="state"):
        T.AdamW([x], state="int8")
    with pytest.raises(TypeError):
        T.AdamW([x.half()])
    with pytest.raises(ValueError):
        T.AdamW([])
