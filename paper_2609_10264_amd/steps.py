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
from . import P, _stream
from .attention import _TYPES, FIELD

_KINDS = {"rms": _lib.MVK_NORM_RMS, "layer": _lib.MVK_NORM_LAYER}
_ACTS = {"silu": _lib.MVK_ACT_SILU, "gelu": _lib.MVK_ACT_GELU, "gelu_tanh": _lib.MVK_ACT_GELU_TANH,
         "relu": _lib.MVK_ACT_RELU}

__all__ = ["Norm", "block_norm", "gated_activation", "sample"]


def _on(t, name: str, device: int):
    """The type of a tensor on the current device."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.device.index != device:
        raise ValueError(f"{name} is on device {t.device.index}, the current device is {device}")
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise TypeError(f"{name} must be bfloat16, float16, float32 or int32 (field), got {t.dtype}")
    return kind


def _matrix(t, name: str, T: int, n: int, device: int):
    """T x n, any stride between rows, contiguous rows."""
    kind = _on(t, name, device)
    if t.dim() != 2 or t.shape[0] != T or t.shape[1] != n:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {(T, n)}")
    a, b = t.stride()
    if b != 1 and n > 1:
        raise ValueError(f"{name}: the last axis must be contiguous")
    return _lib.MvkRows(t.data_ptr(), kind, a, n)


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
        kind, at = _lib.MVK_TYPE_F32, [None, None]
        for i, (t, name) in enumerate(((self.weight, "weight"), (self.bias, "bias"))):
            if t is None:
                continue
            kind = _on(t, name, device)
            if t.shape != (n,) or not t.is_contiguous():
                raise ValueError(f"{name} must be {n} contiguous values, got {tuple(t.shape)}")
            at[i] = t.data_ptr()
        if None not in at and self.weight.dtype != self.bias.dtype:
            raise TypeError("weight and bias must have one type")
        return _lib.MvkNorm(at[0], at[1], kind, _KINDS[self.kind], self.eps)


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
    device = torch.cuda.current_device()
    like = x if x is not None else residual
    if like is None:
        raise ValueError("one of x and residual is needed")
    if like.dim() != 2:
        raise ValueError(f"rows are T x n, got {tuple(like.shape)}")
    T, n = like.shape
    ref = ctypes.byref
    xs = _matrix(x, "x", T, n, device) if x is not None else None
    rs = _matrix(residual, "residual", T, n, device) if residual is not None else None
    stream_type = residual.dtype if residual is not None else torch.float32
    if residual_out is None:
        residual_out = torch.empty((T, n), dtype=stream_type, device=like.device)
    if out is None and (before is not None or out_dtype is not None):
        out = torch.empty((T, n), dtype=out_dtype or stream_type, device=like.device)
    ho = _matrix(residual_out, "residual_out", T, n, device)
    os_ = _matrix(out, "out", T, n, device) if out is not None else None
    gs = None
    if gate is not None:
        kind = _on(gate, "gate", device)
        if gate.dim() == 1:
            if gate.shape[0] != n or (gate.stride(0) != 1 and n > 1):
                raise ValueError(f"gate must be {n} contiguous values or {(T, n)}, got {tuple(gate.shape)}")
            gs = _lib.MvkRows(gate.data_ptr(), kind, 0, n)
        else:
            gs = _matrix(gate, "gate", T, n, device)
    norms = [ref(w.struct(n, device)) if w is not None else None for w in (after, before)]
    _lib.check("mvk_block_norm", _lib.load(p).mvk_block_norm(
        ref(xs) if xs is not None else None, _scale_of(xs.type, field_scale, "field_scale") if xs is not None else 0.0,
        ref(rs) if rs is not None else None, T, n, norms[0], ref(gs) if gs is not None else None, scale, ref(ho),
        norms[1], ref(os_) if os_ is not None else None,
        _scale_of(os_.type, out_scale, "out_scale") if os_ is not None else 0.0, _stream(stream)))
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
    device = torch.cuda.current_device()
    if not isinstance(gate, torch.Tensor) or gate.dim() != 2:
        raise ValueError("gate must be a tensor, T x n")
    T, n = gate.shape
    gs, us = _matrix(gate, "gate", T, n, device), _matrix(up, "up", T, n, device)
    if out is None:
        out_dtype = out_dtype or (torch.float32 if gate.dtype == FIELD else gate.dtype)
        out = torch.empty((T, n), dtype=out_dtype, device=gate.device)
    os_ = _matrix(out, "out", T, n, device)
    ref = ctypes.byref
    _lib.check("mvk_gated_activation", _lib.load(p).mvk_gated_activation(
        ref(gs), ref(us), T, n, _ACTS[act], _scale_of(gs.type, field_scale, "field_scale"), ref(os_),
        _scale_of(os_.type, out_scale, "out_scale"), _stream(stream)))
    return out


def _each(v, name: str, dtype, R: int, device: int):
    """(value for all rows, pointer to one a row)"""
    if not isinstance(v, torch.Tensor):
        return v, None
    if not v.is_cuda or v.dtype != dtype or v.shape != (R,) or not v.is_contiguous():
        raise ValueError(f"{name} must be a number or {R} contiguous CUDA values of {dtype}")
    if v.device.index != device:
        raise ValueError(f"{name} is on device {v.device.index}, the current device is {device}")
    return 0, v.data_ptr()


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
    device = torch.cuda.current_device()
    if not isinstance(logits, torch.Tensor) or logits.dim() != 2:
        raise ValueError("logits must be a tensor, R x n")
    R, n = logits.shape
    rows = _matrix(logits, "logits", R, n, device)
    if out is None:
        out = torch.empty((R,), dtype=torch.int32, device=logits.device)
    at = []
    for t, name, dtype in ((u, "u", torch.float32), (out, "out", torch.int32), (probs, "probs", torch.float32)):
        if t is None and name == "probs":
            at.append(None)
            continue
        _on(t, name, device)
        if t.dtype != dtype or t.shape != (R,) or not t.is_contiguous():
            raise ValueError(f"{name} must be {R} contiguous values of {dtype}")
        at.append(t.data_ptr())
    f32 = torch.float32
    (t, ts), (k, ks), (pp, ps), (m, ms) = (_each(temperature, "temperature", f32, R, device),
                                           _each(top_k, "top_k", torch.int32, R, device),
                                           _each(top_p, "top_p", f32, R, device), _each(min_p, "min_p", f32, R, device))
    how = _lib.MvkSampling(t, pp, m, max(min(k, 2**31 - 1), 0), ts, ps, ms, ks)
    _lib.check("mvk_sample_tokens", _lib.load(p).mvk_sample_tokens(
        ctypes.byref(rows), R, n, _scale_of(rows.type, field_scale, "field_scale"), ctypes.byref(how), *at,
        _stream(stream)))
    return out
