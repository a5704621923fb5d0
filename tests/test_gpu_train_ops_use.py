"""The training operators as a program uses them: optimizers that are copied or share parameters, calls that are refused, tensors that
autograd hands over as it likes, and derivatives of derivatives."""
import copy
import io

import pytest
import torch

from paper_1903_04488_b200 import autograd as A
from paper_1903_04488_b200 import train_ops as T

pytestmark = pytest.mark.gpu

HYPER = dict(lr=1e-2, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)


def rand(*shape, seed=1, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def saved(opt):
    file = io.BytesIO()
    torch.save(opt, file)
    file.seek(0)
    return torch.load(file, weights_only=False)


@pytest.mark.parametrize("again", [copy.deepcopy, saved])
@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_a_copied_optimizer_steps_its_own_tensors(cuda_device, state, again):
    a = T.AdamW([rand(n, seed=n) for n in (1000, 7, 300)], state=state, **HYPER)
    grads = [rand(n, seed=n + 1) for n in (1000, 7, 300)]
    a.step(grads, seed=1)
    b = again(a)
    before = [p.clone() for p in b.params]
    a.step(grads, seed=2)
    assert all(torch.equal(p, q) for p, q in zip(b.params, before)) and b.step_count == 1
    want = [[t.float().clone() for t in x] for x in (a.params, a.m, a.v)]
    del a
    b.step(grads, seed=2)
    assert b.step_count == 2
    assert all(torch.equal(p.float(), q) for x, y in zip((b.params, b.m, b.v), want) for p, q in zip(x, y))


def test_a_second_derivative_is_refused(cuda_device):
    x, w, b = (t.requires_grad_() for t in (rand(6, 32), rand(32, seed=2), rand(32, seed=3)))
    dx, = torch.autograd.grad(A.layer_norm(x, w, b).square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        (dx.square().sum() + x.square().sum()).backward()
    z = rand(6, 32, seed=4).requires_grad_()
    ids = torch.zeros(6, dtype=torch.int64, device="cuda")
    dz, = torch.autograd.grad(A.token_logprobs(z, ids)[0].square().sum(), z, create_graph=True)
    with pytest.raises(RuntimeError):
        (dz.square().sum() + z.square().sum()).backward()


def test_8bit_states_round_stochastically_unless_told_otherwise(cuda_device):
    """A second moment that shrinks by a hundredth a step follows; rounded to nearest it would stay where it is."""
    n = 1 << 16
    opt = T.AdamW([torch.zeros(n, device="cuda")], state="e4m3", betas=(0.9, 0.99), lr=0.0)
    opt.step([torch.rand(n, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda") * 0.1 + 0.01])
    second = lambda: float((opt.v[0].double() * opt.v_scale[0].double().repeat_interleave(256)).square().mean())  # noqa: E731
    v0 = second()
    for _ in range(100):
        opt.step([torch.zeros(n, device="cuda")])
    # every rounding adds at most (value / 16)^2 to the square's mean: 0.99 + 1 / 256 a step
    assert second() < 0.75 * v0
    # the seed of a step is its number
    a, b = (T.AdamW([torch.zeros(n, device="cuda")], state="e4m3") for _ in range(2))
    for t in (1, 2, 3):
        a.step([rand(n, seed=t)])
        b.step([rand(n, seed=t)], seed=t)
    assert torch.equal(a.m[0].float(), b.m[0].float()) and torch.equal(a.v[0].float(), b.v[0].float())
    # states in fp32 round nothing, and bfloat16 parameters to nearest unless a seed is given
    p, q = (rand(n, seed=9, dtype=torch.bfloat16) for _ in range(2))
    T.AdamW([p], **HYPER).step([rand(n, seed=3)])
    T.AdamW([q], **HYPER).step([rand(n, seed=3)], seed=None)
    assert torch.equal(p, q)


def test_tensors_that_share_memory_are_refused(cuda_device):
    p, flat = rand(100), rand(1000)
    for params in ([p, p], [p, rand(5), p.view(10, 10)], [flat[:600], flat[599:]]):
        with pytest.raises(ValueError, match="overlap"):
            T.AdamW(params)
    with pytest.raises(ValueError, match="overlap"):
        T.AdamW([p], m=[p], v=[torch.zeros(100, device="cuda")])
    m = torch.zeros(100, device="cuda")
    with pytest.raises(ValueError, match="overlap"):
        T.AdamW([p], m=[m], v=[m])
    state = torch.zeros(512, dtype=torch.float8_e4m3fn, device="cuda")
    s = torch.zeros(2, device="cuda")
    with pytest.raises(ValueError, match="overlap"):
        T.AdamW([rand(512)], state="e4m3", m=[state], v=[state.clone()], m_scale=[s], v_scale=[s])
    c = torch.zeros(150, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="overlap"):
        T.AdamW([rand(100), rand(100)], copies=[c[:100], c[50:]])
    T.AdamW([flat[:600], flat[600:], flat[:0], flat[:0]]).step([rand(600), rand(400), rand(0), rand(0)])


def test_a_refused_call_leaves_its_tensors_as_they_were(cuda_device):
    """Values and autograd's version counters."""
    p, g = rand(100), rand(100)
    copies = [torch.zeros(100, dtype=torch.bfloat16, device="cuda")]
    opt = T.AdamW([p], copies=copies, **HYPER)
    x, w, stats = rand(8, 64), rand(64), rand(2, 8)
    z, ids = rand(8, 64), torch.zeros(8, dtype=torch.int64, device="cuda")
    out, dw, db = torch.zeros(8, 64, device="cuda"), torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda")
    written = [p, copies[0], out, dw, db] + opt.m + opt.v
    before = [(t._version, t.clone()) for t in written]
    for call in (lambda: opt.step([g], grad_scale=torch.ones(2, device="cuda")), lambda: opt.step([g], seed=1.5), lambda: opt.step([g], lr="x"),
                 lambda: opt.step([g], lr=-1.0), lambda: T.layer_norm(x, w[:3], out=out), lambda: T.layer_norm(x, w, eps=-1.0, out=out),
                 lambda: T.layer_norm(x, w, eps="x", out=out), lambda: T.layer_norm_backward(x, x, w.half(), stats, dx=out, dw=dw, db=db),
                 lambda: T.layer_norm_backward(x, x, w, stats, dx=out, dw=dw, db=db[:5]),
                 lambda: T.token_logprobs_backward(z, ids, z[:, 0].contiguous(), None, scale=0.0, out=out),
                 lambda: T.token_logprobs_backward(z, ids, z[:, 0].contiguous(), None, scale="x", out=out)):
        with pytest.raises((TypeError, ValueError, RuntimeError)):
            call()
    assert opt.step_count == 0
    for t, (version, value) in zip(written, before):
        assert t._version == version and torch.equal(t, value)
    # what is written to does move on
    T.layer_norm(x, w, out=out)
    T.layer_norm_backward(x, x, w, stats, dx=out, dw=dw, db=db)
    T.token_logprobs_backward(z, ids, z[:, 0].contiguous(), None, out=out)
    opt.step([g])
    assert out._version == before[2][0] + 3 and dw._version == before[3][0] + 1 and db._version == before[4][0] + 1
    assert p._version > before[0][0] and copies[0]._version > before[1][0]


def test_autograd_takes_tensors_however_they_lie(cuda_device):
    x, w, b, dy = rand(6, 5, 32), rand(64, seed=2)[::2], rand(64, seed=3)[1::2], rand(6, 5, 32, seed=4)
    for view in (lambda t: t.transpose(0, 1), lambda t: t[:, ::2], lambda t: t[0].t(), lambda t: t[:1].expand(6, 5, 32), lambda t: t[0, :1].expand(5, 32),
                 lambda t: t[:, 1], lambda t: t[0, 0]):
        xv = view(x).detach()
        lies = xv.detach().requires_grad_()
        plain = xv.clone(memory_format=torch.contiguous_format).requires_grad_()
        n = xv.shape[-1]
        params = [(t[:n].detach().requires_grad_() if n <= 32 else None) for t in (w, b)]
        y = A.layer_norm(lies, *params)
        d = view(dy)
        gx, gw, gb = torch.autograd.grad(y, [lies, *params], d)
        y2 = A.layer_norm(plain, params[0].detach().contiguous(), params[1].detach().contiguous())
        want = torch.autograd.grad(torch.nn.functional.layer_norm(plain, (n,), *params, 1e-5), [plain, *params], d)
        assert torch.equal(y, y2)
        for got, ref in zip((gx, gw, gb), want):
            assert got.shape == ref.shape and (got - ref).abs().max() <= 1e-4 * (1 + ref.abs().max())
    z = rand(50, 12)
    for zv in (z.t(), z[:, ::3], z[:1].expand(4, 12)):
        rows = zv.shape[0]
        lies, plain = zv.detach().requires_grad_(), zv.clone(memory_format=torch.contiguous_format).requires_grad_()
        ids = torch.zeros(rows, 2, dtype=torch.int64, device="cuda")[:, 0]
        got, want = A.token_logprobs(lies, ids), A.token_logprobs(plain, ids.contiguous())
        assert torch.equal(got[0], want[0])
        gl, gp = torch.autograd.grad(got[0].sum(), lies), torch.autograd.grad(want[0].sum(), plain)
        assert torch.equal(gl[0], gp[0])


def test_rows_of_one_value_are_normalised_to_zero(cuda_device):
    """The mean of a row of one value is that value wherever the sum is exact: nothing is left to be divided by a small deviation."""
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        for n in (40, 1000, 1030, 2050, 3000, 5000, 7000, 9000, 17000, 40000):
            for rows in (1, 3, 1500):
                if rows * n > 1 << 24:
                    continue
                for value in (3.0, 48.0, 1000.0, 24064.0, 50000.0):
                    if dtype == torch.bfloat16 and value == 1000.0:
                        value = 1008.0
                    x = torch.full((rows, n), value, device="cuda").to(dtype)
                    y, stats = T.layer_norm(x, None, None, 1e-5)
                    assert (stats[0] == x[0, 0].float()).all() and not y.any(), (dtype, rows, n, value, float(stats[0, 0]), float(y.float().abs().max()))
