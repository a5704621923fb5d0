"""Operators of the training step around the compression: layer norm, log probabilities of given tokens, AdamW.

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
