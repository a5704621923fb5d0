"""Operators of the training step around the compression: layer norm, log probabilities of given tokens, AdamW.

The gradient that `Ssgd.step` compresses comes out of a model's layers and loss, and the parameters that are not sketched
need an ordinary optimizer step.  As in `ssgd`, the functions here only check and marshal: the work is done by kernels of
libssgd.so, enqueued on the current stream, and there is no CPU fallback.  `autograd` wraps the differentiable ones.

Rows may have any stride (a piece of a larger tensor will do) as long as the elements of a row are adjacent.  All tensors
of a call are on the current CUDA device.
"""
from __future__ import annotations

import ctypes as C
import functools
import operator

import numpy as np
import torch

from . import ssgd as S

_FMT = {torch.float32: S.FMT_F32, torch.float16: S.FMT_F16, torch.bfloat16: S.FMT_BF16}
_ID_BYTES = {torch.int64: 8, torch.int32: 4}
# the current stream and device, without the objects that torch.cuda's functions make of them
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: torch.cuda.current_stream(dev).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _chk(code: int, what: str) -> None:
    if code:
        raise S.SsgdError(code, what)


def _device(t: torch.Tensor, name: str) -> int:
    if not t.is_cuda:
        raise TypeError(f"{name}: need a CUDA tensor")
    dev = t.get_device()
    if dev != _current_device():
        raise ValueError(f"{name}: on device {dev}, but the current device is {_current_device()}")
    return dev


_PROTO: dict[int, torch.Tensor] = {}


def _f32(dev: int, shape) -> torch.Tensor:
    """An uninitialised float32 tensor (new_empty costs half of what torch.empty with a type and a device does)."""
    proto = _PROTO.get(dev)
    if proto is None:
        proto = _PROTO[dev] = torch.empty(0, dtype=torch.float32, device=f"cuda:{dev}")
    return proto.new_empty(shape)


def _like(t: torch.Tensor) -> torch.Tensor:
    """An uninitialised contiguous tensor of t's shape and type."""
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


@functools.lru_cache(maxsize=1024)
def _norm_workspace(rows: int, n: int) -> int:
    out = S._sz()
    _chk(S.lib().ssgd_layer_norm_backward_workspace(rows, n, C.byref(out)), "ssgd_layer_norm_backward_workspace")
    return out.value


def _rows(t: torch.Tensor, name: str, dev: int | None = None) -> tuple[int, int, int]:
    """(rows, n, stride between rows) of a tensor read as rows of its last dimension."""
    if t.dim() == 2:
        (rows, n), (ld, inner) = t.shape, t.stride()
        if n > 1 and inner != 1:
            raise TypeError(f"{name}: the elements of a row must be adjacent")
        if rows <= 1:
            ld = n
        elif ld < n:
            raise TypeError(f"{name}: rows overlap")
    elif t.dim() > 0 and t.is_contiguous():
        n = t.shape[-1]
        rows, ld = (t.numel() // n if n else 0), n
    else:
        raise TypeError(f"{name}: need a 2-dimensional tensor with adjacent row elements, or a contiguous one")
    if dev is not None and t.get_device() != dev:
        raise TypeError(f"{name}: need a tensor on CUDA device {dev}")
    return rows, n, ld


def _flat(t: torch.Tensor | None, dtype, n: int, name: str, dev: int):
    """Address of a contiguous tensor of n elements (None stays None)."""
    if t is None:
        return None
    if t.dtype != dtype or t.numel() != n or not t.is_contiguous() or t.get_device() != dev:
        raise TypeError(f"{name}: need a contiguous tensor of {n} elements of {dtype} on CUDA device {dev}")
    return t.data_ptr()


def _format(t: torch.Tensor, name: str) -> int:
    fmt = _FMT.get(t.dtype)
    if fmt is None:
        raise TypeError(f"{name}: need float32, float16 or bfloat16")
    return fmt


# ---- layer norm --------------------------------------------------------------------------------------


def layer_norm(x: torch.Tensor, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None, eps: float = 1e-5, *,
               out: torch.Tensor | None = None) -> tuple[torch.Tensor, torch.Tensor]:
    """(y, stats): layer norm over the last dimension of x, and each row's mean and 1 / standard deviation, [2][rows] fp32.

    weight, bias: [n], float32 or x's type, both the same.  out: where y goes (x's shape and type; may be x itself)."""
    dev = _device(x, "x")
    rows, n, ld = _rows(x, "x")
    fmt = _format(x, "x")
    param = weight if weight is not None else bias
    fmt_w = fmt if param is None else _format(param, "weight")
    wp = _flat(weight, param.dtype, n, "weight", dev) if weight is not None else None
    bp = _flat(bias, param.dtype, n, "bias", dev) if bias is not None else None
    if out is None:
        y = _like(x)
        ld_y = n
    else:
        if out.shape != x.shape or out.dtype != x.dtype:
            raise TypeError("out: need x's shape and type")
        y = out
        ld_y = _rows(out, "out", dev)[2]
    stats = _f32(dev, (2, rows))
    _chk(S.lib().ssgd_layer_norm(x.data_ptr(), ld, fmt, wp, bp, fmt_w, rows, n, eps, y.data_ptr(), ld_y, stats.data_ptr(),
                                 _raw_stream(dev)), "ssgd_layer_norm")
    return y, stats


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor | None, stats: torch.Tensor, *,
                        dx: torch.Tensor | None = None, dw: torch.Tensor | None = None, db: torch.Tensor | None = None,
                        accumulate: bool = False, need_params: bool = True):
    """(dx, dw, db) of `layer_norm`; dw and db are float32 [n], None with need_params=False.

    dx, dw, db: where the results go (dx may be dy itself; dw and db may be pieces of a flat gradient).  accumulate adds
    dw and db to what is there."""
    dev = _device(x, "x")
    rows, n, ld = _rows(x, "x")
    fmt = _format(x, "x")
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise TypeError("dy: need x's shape and type")
    ld_dy = _rows(dy, "dy", dev)[2]
    fmt_w = fmt if weight is None else _format(weight, "weight")
    wp = _flat(weight, weight.dtype, n, "weight", dev) if weight is not None else None
    if dx is None:
        dx = _like(x)
        ld_dx = n
    else:
        if dx.shape != x.shape or dx.dtype != x.dtype:
            raise TypeError("dx: need x's shape and type")
        ld_dx = _rows(dx, "dx", dev)[2]
    if need_params:
        if accumulate and (dw is None or db is None):
            raise ValueError("accumulate: needs dw and db")
        if dw is None:
            dw = _f32(dev, (n,))
        if db is None:
            db = _f32(dev, (n,))
    nbytes = _norm_workspace(rows, n)
    ws = _f32(dev, (nbytes // 4,))
    _chk(S.lib().ssgd_layer_norm_backward(dy.data_ptr(), ld_dy, x.data_ptr(), ld, fmt, wp, fmt_w,
                                          _flat(stats, torch.float32, 2 * rows, "stats", dev), rows, n, dx.data_ptr(), ld_dx,
                                          _flat(dw, torch.float32, n, "dw", dev), _flat(db, torch.float32, n, "db", dev),
                                          1 if accumulate else 0, ws.data_ptr(), nbytes, _raw_stream(dev)),
         "ssgd_layer_norm_backward")
    return dx, dw, db


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
    dev = _device(logits, "logits")
    if logits.dim() != 2:
        raise TypeError("logits: need [rows][vocab]")
    rows, vocab, ld = _rows(logits, "logits")
    fmt = _format(logits, "logits")
    id_bytes = _ID_BYTES.get(ids.dtype)
    if id_bytes is None:
        raise TypeError("ids: need int64 or int32")
    ids_p = _flat(ids, ids.dtype, rows, "ids", dev)
    stats = _f32(dev, (3, rows))
    top_idx = top_logp = None
    if top > 0:
        top_idx = torch.empty((rows, top), dtype=torch.int32, device=logits.device)
        top_logp = _f32(dev, (rows, top))
    _chk(S.lib().ssgd_token_logprobs(logits.data_ptr(), ld, fmt, ids_p, id_bytes, rows, vocab, scale, top, stats.data_ptr(),
                                     top_idx.data_ptr() if top > 0 else None, top_logp.data_ptr() if top > 0 else None,
                                     _raw_stream(dev)), "ssgd_token_logprobs")
    return TokenLogprobs(stats, top_idx, top_logp)


def token_logprobs_backward(logits: torch.Tensor, ids: torch.Tensor, lse: torch.Tensor, d_logp: torch.Tensor | None, *,
                            entropy: torch.Tensor | None = None, d_entropy: torch.Tensor | None = None,
                            top_idx: torch.Tensor | None = None, d_top: torch.Tensor | None = None, scale: float = 1.0,
                            out: torch.Tensor | None = None) -> torch.Tensor:
    """Gradient with respect to the logits of sum(d_logp logp) + sum(d_entropy entropy) + sum(d_top top_logp), in the
    logits' type.  lse, entropy, top_idx: from the forward pass with the same scale.  out may be the logits themselves."""
    dev = _device(logits, "logits")
    if logits.dim() != 2:
        raise TypeError("logits: need [rows][vocab]")
    rows, vocab, ld = _rows(logits, "logits")
    fmt = _format(logits, "logits")
    id_bytes = _ID_BYTES.get(ids.dtype)
    if id_bytes is None:
        raise TypeError("ids: need int64 or int32")
    if (top_idx is None) != (d_top is None):
        raise ValueError("top_idx and d_top: give both or neither")
    if d_entropy is not None and entropy is None:
        raise ValueError("d_entropy: needs the forward pass's entropy")
    top = 0
    if top_idx is not None:
        if top_idx.dim() != 2 or top_idx.shape[0] != rows:
            raise TypeError("top_idx: need [rows][top]")
        top = top_idx.shape[1]
    if out is None:
        out = _like(logits)
        ld_out = vocab
    else:
        if out.shape != logits.shape or out.dtype != logits.dtype:
            raise TypeError("out: need the logits' shape and type")
        ld_out = _rows(out, "out", dev)[2]
    f32 = torch.float32
    _chk(S.lib().ssgd_token_logprobs_backward(
        logits.data_ptr(), ld, fmt, _flat(ids, ids.dtype, rows, "ids", dev), id_bytes, rows, vocab, scale,
        _flat(lse, f32, rows, "lse", dev), _flat(entropy, f32, rows, "entropy", dev), _flat(d_logp, f32, rows, "d_logp", dev),
        _flat(d_entropy, f32, rows, "d_entropy", dev), top, _flat(top_idx, torch.int32, rows * top, "top_idx", dev),
        _flat(d_top, f32, rows * top, "d_top", dev), out.data_ptr(), ld_out, _raw_stream(dev)),
        "ssgd_token_logprobs_backward")
    return out


# ---- AdamW over many tensors -------------------------------------------------------------------------

_P, _G, _M, _V, _MS, _VS, _COPY, _N = range(8)     # the fields of ssgd_adamw_tensor, 8 bytes each
_dtype_of = operator.attrgetter("dtype")
_is_none = functools.partial(operator.is_, None)
_numel, _is_contiguous, _get_device, _data_ptr = (torch.Tensor.numel, torch.Tensor.is_contiguous, torch.Tensor.get_device,
                                                  torch.Tensor.data_ptr)


class AdamW:
    """AdamW with decoupled weight decay over a list of contiguous tensors, all of them in one launch per step.

    params: float32, or bfloat16.  state: "f32", or "e4m3" (one byte per element for each of m and sqrt(v), a scale per
    ADAMW_BLOCK elements).  m, v (and m_scale, v_scale for "e4m3"): existing states, one tensor per parameter; fresh zeros
    if None.  copies: for float32 params, bfloat16 or float16 tensors that receive the rounded new values.  step_count: steps
    already taken (with states from a checkpoint)."""

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
        dev = _device(params[0], "params")
        small = state == "e4m3"
        sdtype = torch.float8_e4m3fn if small else torch.float32
        sizes = [p.numel() for p in params]
        blocks = [-(-n // S.ADAMW_BLOCK) for n in sizes]

        def fresh(lens, dt):
            return [torch.zeros(n, dtype=dt, device=params[0].device) for n in lens]

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
        self._dev, self._sizes, self._sizes_u64 = dev, sizes, np.array(sizes, dtype=np.uint64)
        self._desc = np.zeros((len(params), 8), dtype=np.uint64)
        self._desc_p = self._desc.ctypes.data
        self._desc[:, _N] = sizes
        columns = [(_P, params, dtype, sizes, "params"), (_M, self.m, sdtype, sizes, "m"), (_V, self.v, sdtype, sizes, "v")]
        if small:
            columns += [(_MS, self.m_scale, torch.float32, blocks, "m_scale"), (_VS, self.v_scale, torch.float32, blocks, "v_scale")]
        if self.copies is not None:
            columns.append((_COPY, self.copies, self.copies[0].dtype, sizes, "copies"))
        for col, tensors, dt, lens, name in columns:
            if len(tensors) != len(params):
                raise ValueError(f"{name}: need one tensor per parameter")
            self._desc[:, col] = [_flat(t, dt, n, f"{name}[{i}]", dev) for i, (t, n) in enumerate(zip(tensors, lens))]
        self._fmt = (_FMT[dtype], S.FMT_E4M3 if small else S.FMT_F32,
                     S.FMT_BF16 if self.copies is None else _FMT[self.copies[0].dtype])

    def step(self, grads, *, seed: int | None = None, grad_scale: torch.Tensor | None = None, lr: float | None = None) -> None:
        """One step.  grads: one contiguous tensor per parameter (float32, bfloat16 or float16, all the same type), None
        for a parameter that is left alone.  seed: round e4m3 states and bfloat16 parameters stochastically with it (another
        one every step).  grad_scale: float32 scalar on the device that multiplies every gradient."""
        if len(grads) != len(self.params):
            raise ValueError("grads: need one tensor per parameter")
        dev = self._dev
        if dev != _current_device():
            raise ValueError(f"grads: the parameters are on device {dev}, which is not the current one")
        desc, sizes = self._desc, self._sizes
        skipped = any(map(_is_none, grads))
        given = [g for g in grads if g is not None] if skipped else grads
        # what every gradient has to be, checked list by list (a Python statement per tensor would cost more than the launch)
        dtypes = set(map(_dtype_of, given))
        dtype = next(iter(dtypes), torch.float32)
        fmt_g = _FMT.get(dtype)
        if fmt_g is None:
            raise TypeError("grads: need float32, bfloat16 or float16")
        want = [n for g, n in zip(grads, sizes) if g is not None] if skipped else sizes
        if len(dtypes) > 1 or list(map(_numel, given)) != want or not all(map(_is_contiguous, given)) or \
                any(map(dev.__ne__, map(_get_device, given))):
            for i, (g, n) in enumerate(zip(grads, sizes)):
                if g is not None and (g.dtype != dtype or g.numel() != n or not g.is_contiguous() or g.get_device() != dev):
                    raise TypeError(f"grads[{i}]: need a contiguous tensor of {n} elements of {dtype} on CUDA device {dev}")
        if skipped:
            desc[:, _G] = [0 if g is None else g.data_ptr() for g in grads]
            desc[:, _N] = [0 if g is None else n for g, n in zip(grads, sizes)]
        else:
            desc[:, _G] = list(map(_data_ptr, grads))
            desc[:, _N] = self._sizes_u64
        fmt_p, fmt_s, fmt_c = self._fmt
        _chk(S.lib().ssgd_adamw_step(self._desc_p, len(sizes), fmt_p, fmt_g, fmt_s, fmt_c, self.lr if lr is None else lr,
                                     self.betas[0], self.betas[1], self.eps, self.weight_decay, self.step_count + 1,
                                     _flat(grad_scale, torch.float32, 1, "grad_scale", dev), 0 if seed is None else 1,
                                     0 if seed is None else seed & 0xFFFFFFFFFFFFFFFF, _raw_stream(dev)), "ssgd_adamw_step")
        self.step_count += 1
