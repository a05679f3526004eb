"""The client's other nonlinear operations between the delegated projections: the
norms around a block with gate and residual, the gated activation of the
feed-forward part, and the token that answers (mvk_block_norm,
mvk_gated_activation, mvk_sample_tokens in include/mvk.h).

Like attention.py they take decrypted field elements as they are and give the
query of the next projection, so a decoder layer's stream h (T x width floats)
goes through them and the projections without another pass over it:

    x, h = block_norm(None, h, before=Norm(w1), out_dtype=FIELD, out_scale=2**-16)
    ...                                       # q, k, v, attention, o
    x, h = block_norm(yo, h, before=Norm(w2), field_scale=2**-16, out_dtype=FIELD, out_scale=2**-16)
    x = gated_activation(ygate, yup, field_scale=2**-16, out_dtype=FIELD, out_scale=2**-8)
    _, h = block_norm(ydown, h, field_scale=2**-16)
    token = sample(logits, u, temperature=0.8, top_k=50, top_p=0.9)

As in the rest of the binding, every function only checks types and shapes and
passes pointers, strides and the stream.  All tensors are on the current device.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass

import torch

from . import _lib
from . import P
from .attention import _TYPES, FIELD

_KINDS = {"rms": _lib.MVK_NORM_RMS, "layer": _lib.MVK_NORM_LAYER}
_ACTS = {"silu": _lib.MVK_ACT_SILU, "gelu": _lib.MVK_ACT_GELU, "gelu_tanh": _lib.MVK_ACT_GELU_TANH,
         "relu": _lib.MVK_ACT_RELU}

__all__ = ["Norm", "block_norm", "gated_activation", "sample"]


def _on(t, name: str, device: int):
    """The type of a tensor on the current device."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.get_device() != device:
        raise ValueError(f"{name} is on device {t.get_device()}, the current device is {device}")
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise TypeError(f"{name} must be bfloat16, float16, float32 or int32 (field), got {t.dtype}")
    return kind


def _matrix(t, name: str, shape, device: int):
    """T x n, any stride between rows, contiguous rows.  (These checks cost as much as a launch if
    written with loops: the messages are found where one has failed.)"""
    if isinstance(t, torch.Tensor) and t.get_device() == device and t.shape == shape:
        kind = _TYPES.get(t.dtype)
        a, b = t.stride()
        if kind is not None and (b == 1 or shape[1] <= 1):
            return _lib.MvkRows(t.data_ptr(), kind, a, shape[1])
    _on(t, name, device)
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    raise ValueError(f"{name}: the last axis must be contiguous")


def _where(stream):
    """(current device, raw stream)"""
    device = torch._C._cuda_getDevice()
    return device, torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream


def _scale_of(kind: int, scale, name: str) -> float:
    """The value of 1 of field elements; without them it is not used."""
    if kind != _lib.MVK_TYPE_FIELD:
        return 0.0
    if scale is None:
        raise ValueError(f"field elements need {name}, the value of 1")
    return scale


@dataclass
class Norm:
    """A norm over rows of n values: "rms", v / sqrt(mean v^2 + eps) * weight +
    bias, or "layer", the same of v less its mean.  weight, bias: n bfloat16,
    float16 or float32 (one type), or None."""
    weight: torch.Tensor | None = None
    bias: torch.Tensor | None = None
    kind: str = "rms"
    eps: float = 1e-6

    def struct(self, n: int, device: int):
        if self.kind not in _KINDS:
            raise ValueError(f"kind must be one of {sorted(_KINDS)}")
        w, b = self.weight, self.bias
        kind, w_at, b_at = _lib.MVK_TYPE_F32, None, None
        if w is not None:
            kind, w_at = self._vector(w, "weight", n, device)
        if b is not None:
            kind, b_at = self._vector(b, "bias", n, device)
            if w is not None and w.dtype != b.dtype:
                raise TypeError("weight and bias must have one type")
        return _lib.MvkNorm(w_at, b_at, kind, _KINDS[self.kind], self.eps)

    @staticmethod
    def _vector(t, name: str, n: int, device: int):
        kind = _on(t, name, device)
        if t.shape != (n,) or not t.is_contiguous():
            raise ValueError(f"{name} must be {n} contiguous values, got {tuple(t.shape)}")
        return kind, t.data_ptr()


def block_norm(x: torch.Tensor | None, residual: torch.Tensor | None = None, before: Norm | None = None,
               after: Norm | None = None, gate: torch.Tensor | None = None, scale: float = 1.0,
               field_scale: float | None = None, out: torch.Tensor | None = None, out_dtype=None,
               out_scale: float | None = None, residual_out: torch.Tensor | None = None, p: int = P, stream=None):
    """h = residual + scale * gate * after(x) and before(h), in one pass over the
    rows (T x n).  x: the block's result, floats or field elements times
    field_scale (None: h is the residual); gate: n or T x n floats.  Returns
    (before(h), h): h in residual_out (may be residual; by default a new tensor of
    residual's type, float32 without one), before(h) in out (may be x) or of
    out_dtype (residual's by default), FIELD: over out_scale, rounded into the field.
    Without `before`, out and out_dtype only h is computed."""
    device, raw = _where(stream)
    like = x if x is not None else residual
    if like is None:
        raise ValueError("one of x and residual is needed")
    shape = like.shape
    if len(shape) != 2:
        raise ValueError(f"rows are T x n, got {tuple(shape)}")
    T, n = shape
    ref = ctypes.byref
    xs = _matrix(x, "x", shape, device) if x is not None else None
    rs = _matrix(residual, "residual", shape, device) if residual is not None else None
    stream_type = residual.dtype if residual is not None else torch.float32
    if residual_out is None:
        residual_out = torch.empty(shape, dtype=stream_type, device=like.device)
    if out is None and (before is not None or out_dtype is not None):
        out = torch.empty(shape, dtype=out_dtype or stream_type, device=like.device)
    ho = _matrix(residual_out, "residual_out", shape, device)
    os_ = _matrix(out, "out", shape, device) if out is not None else None
    gs = None
    if gate is not None:
        kind = _on(gate, "gate", device)
        if gate.dim() == 1:
            if gate.shape[0] != n or (gate.stride(0) != 1 and n > 1):
                raise ValueError(f"gate must be {n} contiguous values or {(T, n)}, got {tuple(gate.shape)}")
            gs = _lib.MvkRows(gate.data_ptr(), kind, 0, n)
        else:
            gs = _matrix(gate, "gate", shape, device)
    _lib.check("mvk_block_norm", _lib.load(p).mvk_block_norm(
        ref(xs) if xs is not None else None, _scale_of(xs.type, field_scale, "field_scale") if xs is not None else 0.0,
        ref(rs) if rs is not None else None, _lib.count(T), _lib.count(n),
        ref(after.struct(n, device)) if after is not None else None,
        ref(gs) if gs is not None else None, scale, ref(ho), ref(before.struct(n, device)) if before is not None else None,
        ref(os_) if os_ is not None else None,
        _scale_of(os_.type, out_scale, "out_scale") if os_ is not None else 0.0, raw))
    return out, residual_out


def gated_activation(gate: torch.Tensor, up: torch.Tensor, act: str = "silu", field_scale: float | None = None,
                     out: torch.Tensor | None = None, out_dtype=None, out_scale: float | None = None, p: int = P,
                     stream=None) -> torch.Tensor:
    """act(gate) * up (T x n each, floats, or field elements times field_scale).
    act: "silu", "gelu", "gelu_tanh" or "relu".  out may be gate or up; out_dtype:
    gate's by default (float32 for field elements), or FIELD: over out_scale,
    rounded into the field."""
    if act not in _ACTS:
        raise ValueError(f"act must be one of {sorted(_ACTS)}")
    device, raw = _where(stream)
    if not isinstance(gate, torch.Tensor) or gate.dim() != 2:
        raise ValueError("gate must be a tensor, T x n")
    shape = gate.shape
    T, n = shape
    gs, us = _matrix(gate, "gate", shape, device), _matrix(up, "up", shape, device)
    if out is None:
        out_dtype = out_dtype or (torch.float32 if gate.dtype == FIELD else gate.dtype)
        out = torch.empty(shape, dtype=out_dtype, device=gate.device)
    os_ = _matrix(out, "out", shape, device)
    ref = ctypes.byref
    _lib.check("mvk_gated_activation", _lib.load(p).mvk_gated_activation(
        ref(gs), ref(us), _lib.count(T), _lib.count(n), _ACTS[act], _scale_of(gs.type, field_scale, "field_scale"),
        ref(os_), _scale_of(os_.type, out_scale, "out_scale"), raw))
    return out


def _vector(t, name: str, dtype, R: int, device: int):
    if isinstance(t, torch.Tensor) and t.get_device() == device and t.dtype == dtype and t.shape == (R,) and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{name} must be {R} contiguous values of {dtype} on the current device")


def _each(v, name: str, dtype, R: int, device: int):
    """(value for all rows, pointer to one a row)"""
    return (0, _vector(v, name, dtype, R, device)) if isinstance(v, torch.Tensor) else (v, None)


def sample(logits: torch.Tensor, u: torch.Tensor, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0,
           field_scale: float | None = None, out: torch.Tensor | None = None, probs: torch.Tensor | None = None,
           p: int = P, stream=None) -> torch.Tensor:
    """A token (int32) for every row of logits (R x n, floats, or field elements
    times field_scale) from random numbers u (R float32 in [0, 1)).  temperature (0:
    the largest logit), top_k (0: off), top_p (1: off), min_p (0: off): numbers, or
    one a row (R float32; top_k int32).  Kept are the first top_k by logit (ties:
    lowest index), of these the shortest prefix with top_p of their probability, and
    of these the ones with at least min_p of the largest's; among the kept ones the
    token is drawn.  probs (R float32, written): its probability among them.  A row
    without a logit above -inf gives -1."""
    device, raw = _where(stream)
    if not isinstance(logits, torch.Tensor) or logits.dim() != 2:
        raise ValueError("logits must be a tensor, R x n")
    R, n = logits.shape
    rows = _matrix(logits, "logits", logits.shape, device)
    if out is None:
        out = torch.empty((R,), dtype=torch.int32, device=logits.device)
    f32 = torch.float32
    at = (_vector(u, "u", f32, R, device), _vector(out, "out", torch.int32, R, device),
          _vector(probs, "probs", f32, R, device) if probs is not None else None)
    (t, ts), (k, ks), (pp, ps), (m, ms) = (_each(temperature, "temperature", f32, R, device),
                                           _each(top_k, "top_k", torch.int32, R, device),
                                           _each(top_p, "top_p", f32, R, device), _each(min_p, "min_p", f32, R, device))
    how = _lib.MvkSampling(t, pp, m, max(min(k, 2**31 - 1), 0), ts, ps, ms, ks)
    _lib.check("mvk_sample_tokens", _lib.load(p).mvk_sample_tokens(
        ctypes.byref(rows), _lib.count(R), _lib.count(n), _scale_of(rows.type, field_scale, "field_scale"),
        ctypes.byref(how), *at, raw))
    return out
