"""AdamW with 8-bit states over several steps: codes and scales are those of the definition, operation for operation.

What is rounded in one step decides the next one's scales, so a code that differs in its last place once can move a whole block later.
The plain form below rounds every operation to 32 bits by itself, in the order that the header states; nothing is left open, so
nothing may differ."""
import math

import pytest
import torch

from paper_1903_04488_b200 import train_ops as T

pytestmark = pytest.mark.gpu

BLOCK = 256
LR, BETAS, EPS, DECAY = 1e-3, (0.9, 0.95), 1e-8, 0.1


def mix(x):
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def words(seed, tensor, n):
    s = torch.tensor([seed & 0xFFFFFFFF], dtype=torch.int64, device="cuda")
    key = mix((mix(mix(s) ^ (seed >> 32)) + tensor) & 0xFFFFFFFF)
    return mix(torch.arange(n, dtype=torch.int64, device="cuda") ^ key)


def to_codes(x, u):
    """Values of the codes, and the scales, of magnitudes x [blocks][256]."""
    amax = x.amax(1, keepdim=True)
    per_scale = torch.where(amax < 2.0 ** -100, 0.0, torch.ones_like(amax) / amax * 448.0)
    y = x * per_scale
    e = torch.floor(torch.log2(y.double().clamp_min(2.0 ** -6))).float()
    e = torch.where(torch.exp2(e) > y.clamp_min(2.0 ** -6), e - 1, e)     # a logarithm that was rounded up
    unit = torch.exp2(e - 3)
    code = torch.floor(y / unit + u) * unit
    return code.clamp_max(448.0), torch.where(amax < 2.0 ** -100, 0.0, amax * torch.tensor(1 / 448, dtype=torch.float32, device="cuda"))


class Plain:
    def __init__(self, n):
        self.nb = -(-n // BLOCK)
        self.n = n
        self.m, self.v = (torch.zeros(self.nb, BLOCK, device="cuda") for _ in range(2))
        self.ms, self.vs = (torch.zeros(self.nb, 1, device="cuda") for _ in range(2))

    def step(self, g, seed, tensor):
        g = torch.nn.functional.pad(g.float(), (0, self.nb * BLOCK - self.n)).view(self.nb, BLOCK)
        m = (self.m * self.ms) * BETAS[0] + g * (1 - BETAS[0])
        r0 = self.v * self.vs
        v = (r0 * r0) * BETAS[1] + (g * g) * (1 - BETAS[1])
        r = torch.sqrt(v)
        if seed is None:
            um = uv = 0.5
        else:
            w = words(seed, tensor, self.nb * BLOCK).view(self.nb, BLOCK)
            um, uv = ((x.float() * 2.0 ** -16 + 2.0 ** -17) for x in (w & 0xFFFF, w >> 16))
        code, self.ms = to_codes(m.abs(), um)
        self.m = torch.where(m < 0, -code, code)
        code, self.vs = to_codes(r, uv)
        self.v = torch.where(v > 0, code.clamp_min(2.0 ** -9), code)


def dense(n, gen, t):
    return torch.randn(n, generator=gen, device="cuda") * 1e-3


def wide(n, gen, t):
    """Blocks in which most values lie far below the largest, and many are zero: codes of the smallest steps."""
    x = torch.randn(n, generator=gen, device="cuda") * torch.exp2(-torch.randint(0, 26, (n,), generator=gen, device="cuda").float())
    return torch.where(torch.rand(n, generator=gen, device="cuda") < 0.2, 0.0, x)


def large(n, gen, t):
    return torch.randn(n, generator=gen, device="cuda") * 2.0 ** (40 if t % 2 else 20)


def tiny(n, gen, t):
    """Second moments around the smallest normal number of 32 bits, whose roots are not small beside 2^-100."""
    return torch.randn(n, generator=gen, device="cuda") * 2.0 ** -62


@pytest.mark.parametrize("make,sizes,steps,gtype,ptype", [
    (dense, (60_000_000, 17_000_003), 8, torch.bfloat16, torch.bfloat16), (dense, (9_999_999,), 10, torch.float32, torch.float32),
    (wide, (20_000_001, 777, 4_000_000), 8, torch.float32, torch.bfloat16), (large, (1_000_000,), 6, torch.float32, torch.float32),
    (tiny, (1_000_000,), 6, torch.float32, torch.float32)])
@pytest.mark.parametrize("seeded", [True, False])
def test_codes_and_scales_are_the_definitions_over_several_steps(cuda_device, make, sizes, steps, gtype, ptype, seeded):
    if not seeded:
        sizes = tuple(n // 8 + 1 for n in sizes)
    gen = torch.Generator(device="cuda").manual_seed(len(sizes))
    params = [torch.randn(n, generator=gen, device="cuda").to(ptype) for n in sizes]
    opt = T.AdamW(params, state="e4m3", lr=LR, betas=BETAS, eps=EPS, weight_decay=DECAY)
    plain = [Plain(n) for n in sizes]
    for t in range(1, steps + 1):
        grads = [make(n, gen, t).to(gtype) for n in sizes]
        seed = (t << 33 | 5 * t) if seeded else None
        opt.step(grads, seed=seed)
        for i, (q, g) in enumerate(zip(plain, grads)):
            q.step(g, seed, i)
            for name, got, want in (("m_scale", opt.m_scale[i], q.ms), ("v_scale", opt.v_scale[i], q.vs),
                                    ("m", opt.m[i].float(), q.m), ("v", opt.v[i].float(), q.v)):
                bad = int((got != want.reshape(-1)[: got.numel()]).sum())
                assert bad == 0, f"step {t}, tensor {i}: {bad} of {got.numel()} of {name} differ"


def test_a_block_of_what_is_hardly_there_is_held_as_zeros(cuda_device):
    """The largest magnitude below 2^-100: scale 0.  Just above: codes and a scale."""
    for exponent, there in ((-105, False), (-95, True)):
        p = torch.zeros(256, device="cuda")
        opt = T.AdamW([p], state="e4m3", betas=(0.5, 0.5), lr=0.0)
        opt.step([torch.full((256,), 2.0 ** exponent, device="cuda")], seed=1)
        assert bool((opt.m_scale[0] > 0).all()) == there
        if there:
            assert (opt.m[0].float() == 448).all() and math.isclose(float(opt.m_scale[0][0]) * 448, 2.0 ** (exponent - 1), rel_tol=1e-6)


@pytest.mark.parametrize("make", [dense, wide, large])
def test_codes_do_not_depend_on_where_the_tensors_lie(cuda_device, make):
    """The same step on tensors that start anywhere, whose blocks are read element by element."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    n = 200_003
    start = torch.randn(n, generator=gen, device="cuda").to(torch.bfloat16)

    def at(offset, dtype):
        return torch.zeros(n + 16, device="cuda").to(dtype)[offset: offset + n]

    def optimizer(offset):
        p = at(offset, torch.bfloat16)
        p.copy_(start)
        return T.AdamW([p], state="e4m3", m=[at(offset, torch.float8_e4m3fn)], v=[at(offset, torch.float8_e4m3fn)],
                       m_scale=[torch.zeros(-(-n // BLOCK), device="cuda")], v_scale=[torch.zeros(-(-n // BLOCK), device="cuda")])

    a, b = optimizer(0), optimizer(3)
    for t in range(1, 7):
        g = make(n, gen, t)
        there = at(5, torch.float32)
        there.copy_(g)
        a.step([g])
        b.step([there])
        for x, y in ((a.params, b.params), (a.m, b.m), (a.v, b.v), (a.m_scale, b.m_scale), (a.v_scale, b.v_scale)):
            assert torch.equal(x[0].float(), y[0].float())


@pytest.mark.parametrize("make", [dense, wide, large])
def test_what_is_not_finite_leaves_the_others_codes_alone(cuda_device, make):
    """A block's other elements and its scales are what they would be if the gradient were 0 there."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    n = 100_000
    g = make(n, gen, 1)
    bad = torch.rand(n, generator=gen, device="cuda") < 0.003
    values = torch.tensor([math.nan, math.inf, -math.inf], device="cuda")[torch.randint(0, 3, (n,), generator=gen, device="cuda")]
    a, b = (T.AdamW([torch.zeros(n, device="cuda")], state="e4m3") for _ in range(2))
    a.step([torch.where(bad, values, g)])
    b.step([torch.where(bad, 0.0, g)])
    assert torch.equal(a.m_scale[0], b.m_scale[0]) and torch.equal(a.v_scale[0], b.v_scale[0])
    for x, y in ((a.m, b.m), (a.v, b.v), (a.params, b.params)):
        assert torch.equal(x[0].float()[~bad], y[0].float()[~bad])
    assert a.m[0].float()[bad].isnan().all() and a.v[0].float()[bad].isnan().all()
