"""Operators of the training step around the compression: layer norm, log probabilities of given tokens, AdamW; and of fine-tuning: the
policy loss, the preference loss, orthogonalised matrices and Muon.

The gradient that `Ssgd.step` compresses comes out of a model's layers and loss, and the parameters that are not sketched
need an ordinary optimizer step.  The work is done by kernels of libssgd.so, enqueued on the current stream; the checks of
tensors and the marshalling by the native module _train_ops beside it.  There is no CPU fallback: if either has not been
built, the first call raises.  `autograd` wraps the differentiable ones.

Rows may have any stride (a piece of a larger tensor will do) as long as the elements of a row are adjacent.  All tensors
of a call are on the current CUDA device.
"""
from __future__ import annotations

import importlib.machinery
import importlib.util
import os

import numpy as np
import torch

from . import ssgd as S

BINDING_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_train_ops.so")
_native = None


def native():
    """The native module.  Raises if it, or the library, has not been built."""
    global _native
    if _native is None:
        S.lib()
        if not os.path.exists(BINDING_PATH):
            raise RuntimeError(f"{BINDING_PATH} is missing: run `python -m paper_1903_04488_b200.build`")
        loader = importlib.machinery.ExtensionFileLoader("_train_ops", BINDING_PATH)
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_train_ops", loader))
        loader.exec_module(module)
        module.set_error_class(S.SsgdError)
        _native = module
    return _native


# ---- layer norm --------------------------------------------------------------------------------------


def layer_norm(x: torch.Tensor, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None, eps: float = 1e-5, *,
               out: torch.Tensor | None = None) -> tuple[torch.Tensor, torch.Tensor]:
    """(y, stats): layer norm over the last dimension of x, and each row's mean and 1 / standard deviation, [2][rows] fp32.

    weight, bias: [n], float32 or x's type, both the same.  out: where y goes (x's shape and type; may be x itself)."""
    return (_native or native()).layer_norm(x, weight, bias, eps, out)


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor | None, stats: torch.Tensor, *,
                        dx: torch.Tensor | None = None, dw: torch.Tensor | None = None, db: torch.Tensor | None = None,
                        accumulate: bool = False, need_params: bool = True):
    """(dx, dw, db) of `layer_norm`; dw and db are float32 [n], None with need_params=False.

    dx, dw, db: where the results go (dx may be dy itself; dw and db may be pieces of a flat gradient).  accumulate adds
    dw and db to what is there."""
    return (_native or native()).layer_norm_backward(dy, x, weight, stats, dx, dw, db, accumulate, need_params)


# ---- log probabilities of given tokens ---------------------------------------------------------------


class TokenLogprobs:
    """stats [3][rows] fp32 (logp, entropy and lse are its rows); top_idx int32 and top_logp fp32 [rows][top], or None."""
    __slots__ = ("stats", "top_idx", "top_logp")

    def __init__(self, stats, top_idx, top_logp):
        self.stats, self.top_idx, self.top_logp = stats, top_idx, top_logp

    @property
    def logp(self) -> torch.Tensor:
        return self.stats[0]

    @property
    def entropy(self) -> torch.Tensor:
        return self.stats[1]

    @property
    def lse(self) -> torch.Tensor:
        return self.stats[2]


def token_logprobs(logits: torch.Tensor, ids: torch.Tensor, *, top: int = 0, scale: float = 1.0) -> TokenLogprobs:
    """Log probability of ids[row] under softmax(scale * logits[row]), the distribution's entropy, log sum exp and the
    `top` best alternatives.  logits [rows][vocab]; ids [rows] int64 or int32 (outside the vocabulary: ignored)."""
    return TokenLogprobs(*(_native or native()).token_logprobs(logits, ids, top, scale))


def token_logprobs_backward(logits: torch.Tensor, ids: torch.Tensor, lse: torch.Tensor, d_logp: torch.Tensor | None, *,
                            entropy: torch.Tensor | None = None, d_entropy: torch.Tensor | None = None,
                            top_idx: torch.Tensor | None = None, d_top: torch.Tensor | None = None, scale: float = 1.0,
                            out: torch.Tensor | None = None) -> torch.Tensor:
    """Gradient with respect to the logits of sum(d_logp logp) + sum(d_entropy entropy) + sum(d_top top_logp), in the
    logits' type.  lse, entropy, top_idx: from the forward pass with the same scale.  out may be the logits themselves."""
    return (_native or native()).token_logprobs_backward(logits, ids, lse, d_logp, entropy, d_entropy, top_idx, d_top, scale, out)


# ---- losses over log probabilities -------------------------------------------------------------------


class PolicyLoss:
    """stats [5][rows] fp32 (loss, logp, entropy, kl and ratio are its rows); dlogits in the logits' type, or None."""
    __slots__ = ("stats", "dlogits")

    def __init__(self, stats, dlogits):
        self.stats, self.dlogits = stats, dlogits

    @property
    def loss(self) -> torch.Tensor:
        return self.stats[0]

    @property
    def logp(self) -> torch.Tensor:
        return self.stats[1]

    @property
    def entropy(self) -> torch.Tensor:
        return self.stats[2]

    @property
    def kl(self) -> torch.Tensor:
        return self.stats[3]

    @property
    def ratio(self) -> torch.Tensor:
        return self.stats[4]


def policy_loss(logits: torch.Tensor, ids: torch.Tensor, old_logp: torch.Tensor, advantages: torch.Tensor, *,
                ref_logp: torch.Tensor | None = None, weights: torch.Tensor | None = None, clip=(0.2, 0.2), kl: float = 0.0,
                entropy: float = 0.0, scale: float = 1.0, need_grad: bool = True, out: torch.Tensor | None = None) -> PolicyLoss:
    """The clipped policy loss of sampled tokens and, in the same pass, the gradient of its sum with respect to the logits:
    loss = weights (-min(r A, clip(r, 1 - clip[0], 1 + clip[1]) A) + kl K - entropy H), r = e^(logp - old_logp), and with q = ref_logp - logp
    K = e^q - 1 - q, which estimates the divergence from the reference without bias.

    logits [rows][vocab]; ids [rows] int64 or int32; old_logp, advantages, ref_logp, weights: [rows] float32.  For a mean, give weights
    1 / number of tokens.  Rows of weight 0 (padding, prompts) or with an id outside the vocabulary are not read: their statistics and
    gradients are 0.  out: where the gradient goes (may be the logits themselves).  need_grad=False: the statistics only."""
    low, high = clip
    return PolicyLoss(*(_native or native()).policy_loss(logits, ids, old_logp, advantages, ref_logp, weights, low, high, kl, entropy, scale,
                                                         need_grad, out))


class PreferenceLoss:
    """loss [pairs], rewards [2][pairs] (of the preferred sequences and of the others) and d_logp (logp's shape), or None; all fp32."""
    __slots__ = ("loss", "rewards", "d_logp")

    def __init__(self, loss, rewards, d_logp):
        self.loss, self.rewards, self.d_logp = loss, rewards, d_logp


PREFERENCE_KINDS = {"sigmoid": S.PREFERENCE_SIGMOID, "ipo": S.PREFERENCE_IPO, "hinge": S.PREFERENCE_HINGE}


def preference_loss(logp: torch.Tensor, ref_logp: torch.Tensor | None, starts: torch.Tensor, *, beta: float = 0.1,
                    label_smoothing: float = 0.0, kind: str = "sigmoid", average: bool = False, weights: torch.Tensor | None = None,
                    need_grad: bool = True, out: torch.Tensor | None = None) -> PreferenceLoss:
    """The loss of pairs of sequences of which one is preferred, and the gradient of its sum with respect to the tokens' log
    probabilities.  With x = beta (difference of the two sums of logp - ref_logp; with `average` of the means):
    "sigmoid" -(1 - e) log sigmoid(x) - e log sigmoid(-x), e = label_smoothing; "ipo" ((x - 1/2) / beta)^2; "hinge" max(0, 1 - x).

    logp, ref_logp (None: 0): float32, of all tokens (as `token_logprobs` gives them, 0 where there is nothing to predict).  starts:
    int32 or int64 [2 pairs + 1], ascending: sequence s is tokens [starts[s], starts[s + 1]), sequence 2 p the preferred one of pair p.
    weights [pairs].  Tokens of no sequence have gradient 0.  out: where the gradient goes (may be logp itself)."""
    if kind not in PREFERENCE_KINDS:
        raise ValueError('kind: "sigmoid", "ipo" or "hinge"')
    return PreferenceLoss(*(_native or native()).preference_loss(logp, ref_logp, starts, weights, PREFERENCE_KINDS[kind], beta, label_smoothing,
                                                                 average, need_grad, out))


# ---- AdamW over many tensors -------------------------------------------------------------------------

def _check(tensors, dtype, lens, name: str, dev: torch.device) -> None:
    if len(tensors) != len(lens):
        raise ValueError(f"{name}: need one tensor per parameter")
    for i, (t, n) in enumerate(zip(tensors, lens)):
        if t.dtype != dtype or t.numel() != n or not t.is_contiguous() or t.device != dev:
            raise TypeError(f"{name}[{i}]: need a contiguous tensor of {n} elements of {dtype} on {dev}")


def _check_apart(groups) -> None:
    """No two tensors that a step writes to may share memory: different threads have them."""
    spans = sorted((t.data_ptr(), t.numel() * t.element_size(), f"{name}[{i}]")
                   for name, tensors in groups if tensors is not None for i, t in enumerate(tensors) if t.numel())
    for (a, size, first), (b, _, second) in zip(spans, spans[1:]):
        if a + size > b:
            raise ValueError(f"{first} and {second} overlap (give a tensor that several layers share once)")


class AdamW:
    """AdamW with decoupled weight decay over a list of contiguous tensors, all of them in one launch per step.

    params: float32, or bfloat16.  state: "f32", or "e4m3" (one byte per element for each of m and sqrt(v), a scale per
    ADAMW_BLOCK elements).  m, v (and m_scale, v_scale for "e4m3"): existing states, one tensor per parameter; fresh zeros
    if None.  copies: for float32 params, bfloat16 or float16 tensors that receive the rounded new values.  No two of all
    these tensors may share memory.  step_count: steps already taken (with states from a checkpoint)."""

    def __init__(self, params, *, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
                 state: str = "f32", m=None, v=None, m_scale=None, v_scale=None, copies=None, step_count: int = 0):
        params = list(params)
        if state not in ("f32", "e4m3"):
            raise ValueError('state: "f32" or "e4m3"')
        if not params:
            raise ValueError("params: need at least one tensor")
        dtype = params[0].dtype
        if dtype not in (torch.float32, torch.bfloat16):
            raise TypeError("params: need float32 or bfloat16")
        dev = params[0].device
        if dev.type != "cuda":
            raise TypeError("params: need CUDA tensors")
        small = state == "e4m3"
        sdtype = torch.float8_e4m3fn if small else torch.float32
        sizes = [p.numel() for p in params]
        blocks = [-(-n // S.ADAMW_BLOCK) for n in sizes]

        def fresh(lens, dt):
            return [torch.zeros(n, dtype=dt, device=dev) for n in lens]

        if (m is None) != (v is None) or (small and ((m_scale is None) != (m is None) or (v_scale is None) != (m is None))):
            raise ValueError("m, v, m_scale, v_scale: give all of a state or nothing")
        if not small and (m_scale is not None or v_scale is not None):
            raise ValueError("m_scale, v_scale: only with state e4m3")
        self.params = params
        self.m = fresh(sizes, sdtype) if m is None else list(m)
        self.v = fresh(sizes, sdtype) if v is None else list(v)
        self.m_scale = self.v_scale = None
        if small:
            self.m_scale = fresh(blocks, torch.float32) if m_scale is None else list(m_scale)
            self.v_scale = fresh(blocks, torch.float32) if v_scale is None else list(v_scale)
        self.copies = None if copies is None else list(copies)
        if self.copies is not None and (dtype != torch.float32 or self.copies[0].dtype not in (torch.bfloat16, torch.float16)):
            raise TypeError("copies: bfloat16 or float16, and only of float32 params")
        self.lr, self.betas, self.eps, self.weight_decay = lr, tuple(betas), eps, weight_decay
        self.step_count = step_count
        _check(params, dtype, sizes, "params", dev)
        _check(self.m, sdtype, sizes, "m", dev)
        _check(self.v, sdtype, sizes, "v", dev)
        if small:
            _check(self.m_scale, torch.float32, blocks, "m_scale", dev)
            _check(self.v_scale, torch.float32, blocks, "v_scale", dev)
        if self.copies is not None:
            _check(self.copies, self.copies[0].dtype, sizes, "copies", dev)
        _check_apart((("params", params), ("m", self.m), ("v", self.v), ("m_scale", self.m_scale), ("v_scale", self.v_scale),
                      ("copies", self.copies)))
        # room for an ssgd_adamw_tensor (64 bytes) per parameter, and behind them their sizes
        self._buffer = np.zeros(len(params) * 9, dtype=np.int64)
        self._buffer[len(params) * 8:] = sizes
        self._dev = dev.index

    def step(self, grads, *, seed: int | str | None = "step", grad_scale: torch.Tensor | None = None, lr: float | None = None) -> None:
        """One step.  grads: one contiguous tensor per parameter (float32, bfloat16 or float16, all the same type), None
        for a parameter that is left alone.  grad_scale: float32 scalar on the device that multiplies every gradient.

        seed: round e4m3 states and bfloat16 parameters stochastically with it (another one every step); None: to nearest.  "step": with
        e4m3 states the step's number, since their second moment, rounded to nearest, would never move; otherwise None.

        In a CUDA graph a step repeats itself with the lr, step number and seed that it was captured with."""
        if seed == "step":
            seed = None if self.m_scale is None else self.step_count + 1
        (_native or native()).adamw_step(self._buffer, self.params, self.m, self.v, self.m_scale, self.v_scale, self.copies, grads,
                                         self._dev, self.lr if lr is None else lr, *self.betas, self.eps, self.weight_decay,
                                         self.step_count + 1, grad_scale, seed)
        self.step_count += 1


# ---- orthogonalised matrices -------------------------------------------------------------------------

QUINTIC = (3.4445, -4.7750, 2.0315)


def orthogonalize(x: torch.Tensor, *, steps: int = 5, coefficients=QUINTIC, eps: float = 1e-7, products: int | None = None,
                  out: torch.Tensor | None = None) -> torch.Tensor:
    """x / (norm + eps) with the polynomial a s + b s^3 + c s^5 applied to its singular values `steps` times, in x's type: close to
    the nearest matrix with orthonormal rows (or columns), but for singular values that are all but zero.

    x: a matrix (with any row stride), or a contiguous batch of them.  products: 3 for results about as exact as fp32's, 1 for an
    error of about 1e-3 (matrices of less than 512 numbers: up to 7e-3) at a third of the time; None: 1 for bfloat16, otherwise 3.  out: where the result goes (x's shape and type; may be x).
    Waits inside the kernels are bounded; `status` says whether one ran out."""
    a, b, c = coefficients
    return (_native or native()).orthogonalize(x, steps, a, b, c, eps, 0 if products is None else products, out)


class Muon:
    """Momentum, orthogonalised: the optimizer of the matrices beside AdamW for everything else.  All matrices in the same few
    launches per step:  m <- momentum m + (1 - momentum) g,  u = momentum m + (1 - momentum) g (nesterov) or m,
    p <- p (1 - lr weight_decay) - lr scale orthogonalize(u).

    params: contiguous matrices, or batches of them, float32 or bfloat16.  m: existing momenta (float32, of the parameters' shapes);
    fresh zeros if None.  scale: "spectral" (sqrt(max(1, rows / cols)), for weights stored [out][in]), "spectral_t" (sqrt(max(1, cols / rows)),
    for weights stored [in][out], as x @ W takes them), "rms" (0.2 sqrt(max(rows, cols)): updates as large as AdamW's) or a number.  products: as in `orthogonalize`, by the parameters' type.  No two of the tensors may share memory.
    Waits inside the kernels are bounded; `status` says whether one ran out."""

    def __init__(self, params, *, lr: float = 0.02, momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0,
                 steps: int = 5, coefficients=QUINTIC, eps: float = 1e-7, scale: str | float = "spectral", products: int | None = None,
                 m=None):
        params = list(params)
        if not params:
            raise ValueError("params: need at least one tensor")
        dtype, dev = params[0].dtype, params[0].device
        if dtype not in (torch.float32, torch.bfloat16):
            raise TypeError("params: need float32 or bfloat16")
        if dev.type != "cuda":
            raise TypeError("params: need CUDA tensors")
        for i, p in enumerate(params):
            if p.dim() < 2:
                raise TypeError(f"params[{i}]: need a matrix, or a batch of them")
        if scale == "spectral":
            self.scales = [max(1.0, p.shape[-2] / max(1, p.shape[-1])) ** 0.5 for p in params]
        elif scale == "spectral_t":
            self.scales = [max(1.0, p.shape[-1] / max(1, p.shape[-2])) ** 0.5 for p in params]
        elif scale == "rms":
            self.scales = [0.2 * max(p.shape[-2:]) ** 0.5 for p in params]
        elif isinstance(scale, str):
            raise ValueError('scale: "spectral", "spectral_t", "rms" or a number')
        else:
            self.scales = [float(scale)] * len(params)
        self.params = params
        self.m = [torch.zeros_like(p, dtype=torch.float32) for p in params] if m is None else list(m)
        sizes = [p.numel() for p in params]
        _check(params, dtype, sizes, "params", dev)
        _check(self.m, torch.float32, sizes, "m", dev)
        _check_apart((("params", params), ("m", self.m)))
        self.lr, self.momentum, self.nesterov, self.weight_decay = lr, momentum, nesterov, weight_decay
        self.steps, self.coefficients, self.eps, self.products = steps, tuple(coefficients), eps, products
        self._dev = dev.index

    def step(self, grads, *, grad_scale: torch.Tensor | None = None, lr: float | None = None) -> None:
        """One step.  grads: one contiguous tensor per parameter, of its shape (float32, bfloat16 or float16, all the same type), None
        for a parameter that is left alone.  grad_scale: float32 scalar on the device that multiplies every gradient."""
        a, b, c = self.coefficients
        (_native or native()).muon_step(self.params, self.m, self.scales, grads, self._dev, self.lr if lr is None else lr, self.momentum,
                                        self.nesterov, self.weight_decay, self.steps, a, b, c, self.eps,
                                        0 if self.products is None else self.products, grad_scale)


def status() -> None:
    """Waits for the current stream and raises if a wait inside a kernel of these operators has run out since the last call (what it
    wrote is then worthless) or the stream reports an error."""
    (_native or native()).status()
