"""Fine-tuning as a program runs it: the losses, their gradients through a model, and both optimizers together, against the same in 64 bits."""
import pytest
import torch

from paper_1903_04488_b200 import train_lm, train_ops as T

pytestmark = pytest.mark.gpu


@pytest.fixture
def tuner(cuda_device):
    model = train_lm.Model(96, 32, 2, cuda_device, seed=3)
    t = train_lm.Tuner(model)
    g = torch.Generator(device="cuda").manual_seed(1)
    with torch.no_grad():
        for p in model.matrices:               # the policy has left the reference
            p.mul_(1.0 + 0.02 * torch.rand(p.shape, generator=g, device="cuda"))
    cur, sampled, chosen = (torch.randint(0, 96, (80,), generator=g, device="cuda") for _ in range(3))
    return t, cur, sampled, chosen, torch.randn(80, generator=g, device="cuda")


def leaves(model):
    return [*model.matrices, *model.small]


def plain_logits(model, values, cur):
    """The model's formula over 64-bit copies of its parameters."""
    mats, small = values[: len(model.matrices)], values[len(model.matrices):]
    norm = lambda x, w, b: (x - x.mean(-1, keepdim=True)) * (x.var(-1, correction=0, keepdim=True) + 1e-5).rsqrt() * w + b  # noqa: E731
    x = mats[0][cur]
    for i in range(model.layers):
        w, b, b1, b2 = small[4 * i: 4 * i + 4]
        x = x + torch.relu(norm(x, w, b) @ mats[1 + 2 * i] + b1) @ mats[2 + 2 * i] + b2
    return norm(x, *small[-2:]) @ mats[-1]


def gradients_match(model, loss_of):
    values = [p.detach().double().requires_grad_() for p in leaves(model)]
    loss_of(values).backward()
    for p, v in zip(leaves(model), values):
        # matrix products of torch in fp32, chains of some hundred roundings
        assert float((p.grad.double() - v.grad).norm()) <= 2e-5 * float(v.grad.norm()) + 1e-9


def test_policy_gradients_reach_the_parameters(tuner):
    t, cur, sampled, _, adv = tuner
    m = t.model
    with torch.no_grad():
        at = T.token_logprobs(m.logits(cur), sampled).logp
    old = at - 0.1 * torch.sign(adv) * (torch.arange(80, device="cuda") % 5).float()      # 0 to 0.4, some of them clipped, none at a border
    r = t.policy(cur, sampled, old, adv)
    assert r.stats.isfinite().all()

    def loss_of(values):
        lp = torch.log_softmax(plain_logits(m, values, cur), -1)
        ref = torch.log_softmax(plain_logits(m, [p.detach().double() for p in leaves(t.reference)], cur), -1)
        logp, ref = (x.gather(1, sampled[:, None]).squeeze(1) for x in (lp, ref))
        ratio, q = (logp - old.double()).exp(), ref - logp
        surrogate = torch.minimum(ratio * adv.double(), ratio.clamp(0.8, 1.2) * adv.double())
        return (-surrogate + 0.05 * (q.exp() - 1 - q) + 0.001 * (lp.exp() * lp).sum(-1)).mean()

    gradients_match(m, loss_of)


def test_preference_gradients_reach_the_parameters(tuner):
    t, cur, sampled, chosen, _ = tuner
    m = t.model
    loss = t.preference(cur, chosen, sampled)

    def loss_of(values):
        def delta(ids):
            lp = [torch.log_softmax(plain_logits(m, v, cur), -1).gather(1, ids[:, None]).view(-1, 8).sum(1)
                  for v in (values, [p.detach().double() for p in leaves(t.reference)])]
            return lp[0] - lp[1]
        return -torch.nn.functional.logsigmoid(0.5 * (delta(chosen) - delta(sampled))).mean()

    gradients_match(m, loss_of)
    values = [p.detach().double() for p in leaves(m)]
    assert abs(float(loss) - float(loss_of(values))) < 1e-5


def test_both_optimizers_step_together(tuner):
    t, cur, sampled, chosen, adv = tuner
    m = t.model
    t.preference(cur, chosen, sampled)
    before = [p.detach().clone() for p in leaves(m)]
    grads = [p.grad.clone() for p in leaves(m)]
    with torch.no_grad():
        t.step()
    T.status()
    for i, (p, b, g) in enumerate(zip(leaves(m), before, grads)):
        if 0 < i < len(m.matrices) - 1:
            want = b.double() - 5e-3 * max(1.0, p.shape[0] / p.shape[1]) ** 0.5 * train_step_of(g)
            tol = 5e-3 * 1e-4
        else:
            want = b.double() - 2e-3 * g.double() / (g.double().abs() + 1e-8)         # AdamW's first step
            tol = 2e-3 * 1e-3
        assert ((p.double() - want).abs() <= tol + 2.0 ** -23 * b.abs()).all(), i
        assert p.grad is None


def train_step_of(g, momentum=0.95):
    a, b, c = T.QUINTIC
    u = g.double() * (1 - momentum) * (1 + momentum)
    x = u / (u.norm() + 1e-7)
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    for _ in range(5):
        k = x @ x.t()
        x = a * x + (b * k + c * k @ k) @ x
    return x.t() if tall else x


@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_tuning_runs(cuda_device, loss):
    report = train_lm.train(steps=3, workers=2, vocab=64, dim=32, layers=1, tokens=128, report_every=1, quiet=True, tune_steps=3, tune_loss=loss)
    assert len(report) == 3 and all(x == x for row in report for x in row)
    with pytest.raises(ValueError):
        train_lm.tune(None, None, None, 1, 1, "none")


def test_a_backward_pass_of_the_losses_in_a_graph(cuda_device):
    g = torch.Generator(device="cuda").manual_seed(5)
    w = torch.randn(24, 700, generator=g, device="cuda")
    h = torch.randn(40, 24, generator=g, device="cuda")
    ids = torch.randint(0, 700, (40,), generator=g, device="cuda")
    old, adv = torch.full((40,), -6.5, device="cuda"), torch.randn(40, generator=g, device="cuda")
    from paper_1903_04488_b200 import autograd as A

    def loss(x):
        return A.policy_loss(h @ x, ids, old, adv)[0].sum()

    want, = torch.autograd.grad(loss(w.requires_grad_()), w)
    leaf = w.detach().clone().requires_grad_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(loss(leaf), leaf)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, = torch.autograd.grad(loss(leaf), leaf)
    graph.replay()
    assert torch.equal(got, want)
