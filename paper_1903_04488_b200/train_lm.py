"""A small language model trained by simulated data-parallel workers on one GPU: the operators around the compression step
and the step itself, together.

    python -m paper_1903_04488_b200.train_lm [--steps 150] [--workers 4] [--state e4m3] [--tune 20 --tune-loss policy] ...

Every worker computes the gradient of its own batch: a residual network over token embeddings whose norms are
`autograd.layer_norm` and whose loss is `autograd.token_logprobs`.  The matrices live in one flat vector, and their
gradients arrive in the worker's row of g [W][d] directly.  `Ssgd.step` compresses the rows to k coordinates (momentum, error
accumulation, sketch, second round); the model moves along these.  Biases and norm weights are not sketched (the paper
leaves bias terms uncompressed, Section 5): their gradients are averaged and `train_ops.AdamW` takes them in one launch.

The data is synthetic: the next token is a fixed permutation of the current one, or, one time in ten, any token.

`tune` goes on from there as fine-tuning does, on one worker and without compression: the model's own samples are rewarded where they
are the permutation's token (`train_ops.policy_loss`, with the trained model as the reference), or compared with it in pairs
(`autograd.preference_loss`); `train_ops.Muon` takes the blocks' matrices and AdamW everything else.
"""
from __future__ import annotations

import argparse
import copy
import math

import torch

from . import autograd, ssgd, train_ops


class Model:
    """Embedding, `layers` residual blocks (norm, two matrices with a bias each), norm, output matrix."""

    def __init__(self, vocab: int, dim: int, layers: int, device, seed: int = 0):
        gen = torch.Generator().manual_seed(seed)
        shapes = [(vocab, dim)] + [(dim, 2 * dim), (2 * dim, dim)] * layers + [(dim, vocab)]
        self.d = sum(a * b for a, b in shapes)
        self.ld = (self.d + 3) // 4 * 4
        self.theta = torch.zeros(self.ld, device=device)           # the sketched parameters, one flat vector
        self.slices, at = [], 0
        for a, b in shapes:
            self.theta[at: at + a * b] = (torch.randn(a * b, generator=gen) / math.sqrt(a if a != vocab else 1)).to(device)
            self.slices.append((at, (a, b)))
            at += a * b
        self.matrices = [t.requires_grad_() for t in self.views(self.theta)]
        # a norm and two biases to a block, a norm at the end: what is not sketched
        self.small = []
        for _ in range(layers):
            self.small += [torch.ones(dim), torch.zeros(dim), torch.zeros(2 * dim), torch.zeros(dim)]
        self.small += [torch.ones(dim), torch.zeros(dim)]
        self.small = [t.to(device).requires_grad_() for t in self.small]
        self.layers = layers

    def views(self, flat: torch.Tensor):
        return [flat[at: at + a * b].view(a, b) for at, (a, b) in self.slices]

    def logits(self, tokens: torch.Tensor) -> torch.Tensor:
        x = self.matrices[0][tokens]
        for i in range(self.layers):
            w, b, b1, b2 = self.small[4 * i: 4 * i + 4]
            h = torch.relu(autograd.layer_norm(x, w, b) @ self.matrices[1 + 2 * i] + b1)
            x = x + h @ self.matrices[2 + 2 * i] + b2
        return autograd.layer_norm(x, *self.small[-2:]) @ self.matrices[-1]


def batch(vocab: int, n: int, perm: torch.Tensor, gen: torch.Generator):
    cur = torch.randint(0, vocab, (n,), generator=gen, device=perm.device)
    noise = torch.rand(n, generator=gen, device=perm.device) < 0.1
    return cur, torch.where(noise, torch.randint(0, vocab, (n,), generator=gen, device=perm.device), perm[cur])


def train(steps: int = 150, workers: int = 4, vocab: int = 256, dim: int = 64, layers: int = 2, tokens: int = 1024,
          lr: float = 0.1, rho: float = 0.9, small_lr: float = 3e-3, state: str = "f32", report_every: int = 25, quiet: bool = False,
          tune_steps: int = 0, tune_loss: str = "policy"):
    """Returns [(step, mean loss, mean entropy, share of tokens that are the model's best)] at the reported steps.  tune_steps: `tune`
    the model afterwards."""
    device = torch.device("cuda", torch.cuda.current_device())
    model = Model(vocab, dim, layers, device)
    W, d = workers, model.d
    k = max(1, d // 10)
    ncand = min(d, 2 * k)
    eng = ssgd.Ssgd(d, 5, 1 << max(10, (d // 8).bit_length()), k, W, seed=7)
    u, v = (torch.zeros((W, model.ld), device=device) for _ in range(2))
    eng.bind(u, v, ncand)
    opt = train_ops.AdamW(model.small, lr=small_lr, betas=(0.9, 0.99), weight_decay=0.0, state=state)
    g = torch.zeros((W, model.ld), device=device)
    out_idx, out_val = torch.empty(k, dtype=torch.int32, device=device), torch.empty(k, device=device)
    gen = torch.Generator(device=device).manual_seed(1)
    perm = torch.randperm(vocab, generator=gen, device=device)
    share = torch.full((1,), 1.0 / W, device=device)                # the workers' small gradients are averaged
    report = []
    for step in range(steps):
        g.zero_()
        for p in model.small:
            p.grad = None
        sums = torch.zeros(3, device=device)
        for w in range(W):
            for p, grad in zip(model.matrices, model.views(g[w])):
                p.grad = grad                                       # backward adds the gradient to the worker's row
            cur, nxt = batch(vocab, tokens, perm, gen)
            logp, entropy, _, best, _ = autograd.token_logprobs(model.logits(cur), nxt, top=1)
            (-logp.mean()).backward()
            sums += torch.stack([-logp.mean(), entropy.mean(), (best[:, 0] == nxt).float().mean()]).detach()
        with torch.no_grad():
            eng.step(g, rho, ncand, out_idx, out_val)
            model.theta.index_add_(0, out_idx, out_val, alpha=-lr / W)
            opt.step([p.grad for p in model.small], seed=step if state == "e4m3" else None, grad_scale=share)
        if step % report_every == 0 or step == steps - 1:
            report.append((step, *(sums / W).tolist()))
            if not quiet:
                print("step %4d  loss %.4f  entropy %.4f  best token right %.3f" % report[-1])
    if eng.status() != ssgd.OK:
        raise RuntimeError("the compression step reported an error")
    eng.flush()
    if tune_steps:
        tune(model, perm, gen, tune_steps, tokens, tune_loss, quiet=quiet)
    return report


class Tuner:
    """What `tune` keeps: the reference, and an optimizer for the blocks' matrices and one for the rest.  matrix_scale: how the matrices'
    updates are scaled.  The model stores them [in][out], for which it is "spectral_t"; the default is that of `train_ops.Muon`."""

    def __init__(self, model: Model, lr: float = 2e-3, matrix_lr: float = 5e-3, matrix_scale: str | float = "spectral"):
        self.model, self.reference = model, copy.deepcopy(model)
        self.blocks = model.matrices[1:-1]
        self.rest = [model.matrices[0], model.matrices[-1], *model.small]
        self.muon = train_ops.Muon(self.blocks, lr=matrix_lr, scale=matrix_scale) if self.blocks else None
        self.adamw = train_ops.AdamW(self.rest, lr=lr, weight_decay=0.0)

    def policy(self, cur, sampled, old_logp, advantages, kl: float = 0.05):
        """Gradients of the clipped policy loss of sampled tokens; its statistics."""
        with torch.no_grad():
            ref = train_ops.token_logprobs(self.reference.logits(cur), sampled).logp
        logits = self.model.logits(cur)
        r = train_ops.policy_loss(logits.detach(), sampled, old_logp, advantages, ref_logp=ref, weights=torch.full_like(ref, 1.0 / ref.numel()),
                                  kl=kl, entropy=0.001)
        logits.backward(r.dlogits)
        return r

    def preference(self, cur, chosen, rejected, length: int = 8, beta: float = 0.5):
        """Gradients of the preference loss of pairs of `length` tokens; the mean loss."""
        n = cur.numel() // length * length
        inputs = cur[:n].view(-1, 1, length).expand(-1, 2, length).reshape(-1)
        ids = torch.stack([chosen[:n].view(-1, length), rejected[:n].view(-1, length)], 1).reshape(-1)
        starts = torch.arange(0, 2 * n + 1, length, device=cur.device)
        with torch.no_grad():
            ref = train_ops.token_logprobs(self.reference.logits(inputs), ids).logp
        loss, _ = autograd.preference_loss(autograd.token_logprobs(self.model.logits(inputs), ids)[0], ref, starts, beta=beta)
        loss.mean().backward()
        return loss.mean().detach()

    def step(self):
        if self.muon is not None:
            self.muon.step([p.grad for p in self.blocks])
        self.adamw.step([p.grad for p in self.rest])
        for p in [*self.blocks, *self.rest]:
            p.grad = None


def tune(model: Model, perm: torch.Tensor, gen: torch.Generator, steps: int, tokens: int, loss: str = "policy", updates: int = 2, quiet: bool = False):
    """Returns the share of sampled tokens that were the permutation's, at each step."""
    if loss not in ("policy", "preference"):
        raise ValueError('loss: "policy" or "preference"')
    tuner = Tuner(model, matrix_scale="spectral_t")
    for p in [*tuner.blocks, *tuner.rest]:
        p.grad = None                                               # it was a piece of the workers' rows
    shares = []
    for step in range(steps):
        cur, _ = batch(perm.numel(), tokens, perm, gen)
        with torch.no_grad():
            logits = model.logits(cur)
            sampled = torch.multinomial(torch.softmax(logits, -1), 1, generator=gen).squeeze(1)
            old_logp = train_ops.token_logprobs(logits, sampled).logp
            reward = (sampled == perm[cur]).float()
        shares.append(reward.mean())
        for _ in range(updates):
            if loss == "policy":
                tuner.policy(cur, sampled, old_logp, reward - reward.mean())
            else:
                tuner.preference(cur, perm[cur], sampled)
            with torch.no_grad():
                tuner.step()
    train_ops.status()
    shares = torch.stack(shares).tolist() if shares else []
    if shares and not quiet:
        print("tuned: samples right %.3f -> %.3f" % (shares[0], shares[-1]))
    return shares


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=150)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--vocab", type=int, default=256)
    ap.add_argument("--dim", type=int, default=64)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--tokens", type=int, default=1024, help="tokens per worker and step")
    ap.add_argument("--lr", type=float, default=0.1)
    ap.add_argument("--state", choices=("f32", "e4m3"), default="f32", help="how AdamW holds its states")
    ap.add_argument("--tune", type=int, default=0, help="steps of fine-tuning afterwards")
    ap.add_argument("--tune-loss", choices=("policy", "preference"), default="policy")
    a = ap.parse_args()
    train(a.steps, a.workers, a.vocab, a.dim, a.layers, a.tokens, a.lr, state=a.state, tune_steps=a.tune, tune_loss=a.tune_loss)


if __name__ == "__main__":
    main()
