"""What the losses, the orthogonalised matrices and the Muon step refuse, before anything is launched: no GPU is needed (addresses that are
only compared, never read)."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_1903_04488_b200 import build as B
from paper_1903_04488_b200 import ssgd as S
from paper_1903_04488_b200 import train_ops as T

P = 1 << 12                                    # an aligned address
F, D = C.c_float, C.c_double
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def lib():
    B.build()
    return S.lib()


def call(fn, good, **bad):
    kw = dict(good)
    kw.update(bad)
    return fn(*kw.values())


def test_policy_loss_refuses(lib):
    good = dict(z=P, ld=100, fmt=S.FMT_F16, ids=P, id_bytes=8, rows=3, vocab=100, scale=F(1), old=P, adv=P, ref=P, w=P, low=F(0.2), high=F(0.2),
                kl=F(0.1), entropy=F(0.01), stats=P, out=P, ld_out=100, stream=None)
    f = lib.ssgd_policy_loss
    for bad in (dict(z=None), dict(ids=None), dict(old=None), dict(adv=None), dict(ref=None), dict(stats=None), dict(ld=99), dict(ld_out=99),
                dict(vocab=0), dict(vocab=(1 << 27) + 1, ld=1 << 28, ld_out=1 << 28), dict(rows=-1), dict(id_bytes=2), dict(fmt=3), dict(fmt=-1),
                dict(scale=F(0)), dict(scale=F(INF)), dict(scale=F(NAN)), dict(low=F(-0.1)), dict(low=F(1.1)), dict(low=F(NAN)), dict(high=F(-1)),
                dict(high=F(NAN)), dict(kl=F(-1)), dict(kl=F(INF)), dict(kl=F(NAN)), dict(entropy=F(NAN)), dict(entropy=F(INF))):
        assert call(f, good, **bad) == S.EINVAL, bad
    for bad in (dict(z=P + 1), dict(ids=P + 4), dict(out=P + 1), dict(old=P + 2), dict(adv=P + 2), dict(ref=P + 1), dict(w=P + 2), dict(stats=P + 2)):
        assert call(f, good, **bad) == S.EALIGN, bad
    assert call(f, good, rows=0, z=None, ids=None, stats=None, out=None) == S.OK


def test_preference_loss_refuses(lib):
    need = S._sz()
    size = lib.ssgd_preference_loss_workspace
    # two numbers of 64 bits for each pair and one for each 8192 tokens begun, which one CTA takes: 10000 tokens are two of these
    assert size(10000, 7, C.byref(need)) == S.OK and need.value >= 8 * (2 + 14)
    for a in ((-1, 0), (0, -1), ((1 << 40) + 1, 0), (0, (1 << 30) + 1)):
        assert size(*a, C.byref(need)) == S.EINVAL
    assert size(1, 1, None) == S.EINVAL
    size(10000, 7, C.byref(need))
    good = dict(logp=P, ref=P, tokens=10000, starts=P, bytes=4, pairs=7, w=P, kind=0, beta=F(0.1), smoothing=F(0.1), average=0, loss=P, rewards=P, d=P,
                ws=P, ws_bytes=need.value, stream=None)
    f = lib.ssgd_preference_loss
    for bad in (dict(logp=None), dict(starts=None), dict(loss=None), dict(rewards=None), dict(tokens=-1), dict(pairs=-1), dict(bytes=2), dict(kind=3),
                dict(kind=-1), dict(beta=F(0)), dict(beta=F(-1)), dict(beta=F(INF)), dict(beta=F(NAN)), dict(smoothing=F(-0.1)),
                dict(smoothing=F(0.6)), dict(smoothing=F(NAN)), dict(kind=1), dict(kind=2)):
        assert call(f, good, **bad) == S.EINVAL, bad
    for bad in (dict(logp=P + 2), dict(ref=P + 1), dict(starts=P + 2), dict(starts=P + 4, bytes=8), dict(w=P + 2), dict(loss=P + 1), dict(rewards=P + 2),
                dict(d=P + 1), dict(ws=P + 4)):
        assert call(f, good, **bad) == S.EALIGN, bad
    for bad in (dict(ws=None), dict(ws_bytes=need.value - 1)):
        assert call(f, good, **bad) == S.EWORKSPACE, bad
    assert call(f, good, tokens=0, pairs=0, logp=None, starts=None, ws=None) == S.OK


def matrices(*rows):
    """ssgd_matrix: out, in, m, ld_out, ld_in, rows, cols, scale"""
    out = np.zeros((len(rows), 8), dtype=np.int64)
    for i, r in enumerate(rows):
        one = dict(out=P, x=P, m=P, ld_out=700, ld_in=700, rows=300, cols=700)
        one.update(r)
        out[i, :7] = list(one.values())
        out[i, 7] = np.float64(1.0).view(np.int64)
    return out


def test_orthogonalize_and_muon_refuse(lib):
    need = S._sz()

    def size(d, fmt=S.FMT_F32, products=0):
        return lib.ssgd_orthogonalize_workspace(d.ctypes.data, len(d), fmt, products, C.byref(need))

    d = matrices({}, {})
    assert size(d) == S.OK
    three = need.value
    assert size(d, products=1) == S.OK and 8 * 2 * 300 * 700 <= need.value < three
    for bad in (dict(rows=-1), dict(cols=-1), dict(rows=(1 << 20) + 1), dict(cols=(1 << 20) + 1)):
        assert size(matrices(bad)) == S.EINVAL, bad
    for bad in (dict(rows=1 << 20, cols=8192), dict(rows=32769, cols=32769)):
        assert size(matrices(bad)) == S.ETOOBIG, bad
    assert size(d, fmt=7) == S.EINVAL and size(d, products=2) == S.EINVAL
    assert lib.ssgd_orthogonalize_workspace(d.ctypes.data, 2, 2, 0, None) == S.EINVAL
    assert size(matrices(dict(rows=128, cols=256), dict(rows=256, cols=1))) == S.OK and need.value == 0     # small ones need none
    # the workspace of many matrices is that of the largest group of them
    assert size(matrices(*[{}] * 224)) == S.OK
    full = need.value
    assert size(matrices(*[{}] * 700)) == S.OK and need.value == full

    good = dict(count=1, fmt=S.FMT_BF16, products=0, steps=5, a=D(3.4445), b=D(-4.775), c=D(2.0315), eps=D(1e-7), ws=P, ws_bytes=1 << 30, stream=None)

    def ortho(row=None, **bad):
        m = matrices(row or {})
        return call(lambda *a: lib.ssgd_orthogonalize(m.ctypes.data, *a), good, **bad)

    for bad in (dict(count=-1), dict(fmt=S.FMT_E4M3), dict(products=2), dict(steps=0), dict(steps=33), dict(a=D(NAN)), dict(a=D(9)), dict(b=D(50)),
                dict(eps=D(-1)), dict(eps=D(NAN)), dict(eps=D(INF))):
        assert ortho(**bad) == S.EINVAL, bad
    for row in (dict(out=0), dict(x=0), dict(ld_out=699), dict(ld_in=699), dict(rows=-1)):
        assert ortho(row) == S.EINVAL, row
    for row in (dict(out=P + 1), dict(x=P + 1)):
        assert ortho(row) == S.EALIGN, row
    assert ortho(ws=None) == S.EWORKSPACE and ortho(ws_bytes=100) == S.EWORKSPACE and ortho(ws=P + 8) == S.EALIGN
    assert ortho(count=0) == S.OK and ortho(dict(rows=0, out=0, x=0)) == S.OK and ortho(dict(cols=0)) == S.OK

    good = dict(count=1, fp=S.FMT_F32, fg=S.FMT_BF16, products=0, lr=D(0.02), mu=D(0.9), nesterov=1, wd=D(0.1), steps=5, a=D(3.4445), b=D(-4.775),
                c=D(2.0315), eps=D(1e-7), gs=None, ws=P, ws_bytes=1 << 30, stream=None)

    def muon(row=None, **bad):
        m = matrices(row or {})
        return call(lambda *a: lib.ssgd_muon_step(m.ctypes.data, *a), good, **bad)

    for bad in (dict(fp=S.FMT_F16), dict(fg=S.FMT_E4M3), dict(lr=D(-1)), dict(lr=D(NAN)), dict(lr=D(INF)), dict(mu=D(1.0)), dict(mu=D(-0.1)),
                dict(mu=D(NAN)), dict(wd=D(-1)), dict(wd=D(NAN)), dict(steps=0), dict(products=5)):
        assert muon(**bad) == S.EINVAL, bad
    assert muon(dict(m=0)) == S.EINVAL and muon(dict(m=P + 2)) == S.EALIGN and muon(gs=P + 2) == S.EALIGN and muon(dict(out=P + 2)) == S.EALIGN


def test_python_checks_name_the_argument():
    x = torch.zeros(4, 8)
    ids = torch.zeros(4, dtype=torch.int64)
    for f, name in ((lambda: T.policy_loss(x, ids, x[:, 0], x[:, 0]), "logits"), (lambda: T.orthogonalize(x), "x"), (lambda: T.Muon([x]), "params"),
                    (lambda: T.preference_loss(x[0], None, ids), "logp")):
        with pytest.raises(TypeError, match=name):
            f()
    with pytest.raises(ValueError, match="kind"):
        T.preference_loss(x[0], None, ids, kind="none")
    with pytest.raises(ValueError):
        T.Muon([])
