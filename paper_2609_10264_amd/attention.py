"""The client's attention between the delegated projections: rotary positions
with the append to a paged cache, attention over it, and eviction from it
(mvk_rotary_*, mvk_cache_read, mvk_paged_attention, mvk_cache_evict in include/mvk.h).

Decrypted queries, keys and values are field elements of fixed-point numbers;
rotary_append takes them as they are (field_scale: the value of 1) and leaves
floats in the cache, and paged_attention gives its result as floats or again as
field elements, the query of the next projection:

    rot = rotary_table(128, 32768)
    cache = KVCache.allocate(pages, kv_heads, 64, 128)       # one a layer
    seqs = Sequences(table, lens, q_start, max_new=1)        # shared by the layers
    q = rotary_append(yq, yk, yv, positions, rot, cache, seqs, field_scale=2**-16)
    x = paged_attention(q, cache, seqs, out_dtype=FIELD, field_scale=2**-8)

A cache may be held in 8 bits (dtype=torch.float8_e4m3fn or torch.int8, with one
power of two an entry and head): rotary_append then writes codes and exponents, and
attention, eviction and cache_read take them as they are, at half the bytes.

As in the rest of the binding, every function only checks types and shapes and
passes pointers, strides and the stream.
"""
from __future__ import annotations

import ctypes
from contextlib import nullcontext
from dataclasses import dataclass

import torch

from . import _lib
from . import P, _dev, _stream

FIELD = torch.int32  # field elements, as everywhere in this package

_TYPES = {torch.bfloat16: _lib.MVK_TYPE_BF16, torch.float16: _lib.MVK_TYPE_F16, torch.float32: _lib.MVK_TYPE_F32,
          torch.int32: _lib.MVK_TYPE_FIELD}
_CACHE_TYPES = {torch.bfloat16: _lib.MVK_TYPE_BF16, torch.float16: _lib.MVK_TYPE_F16, torch.float32: _lib.MVK_TYPE_F32,
                torch.float8_e4m3fn: _lib.MVK_TYPE_E4M3, torch.int8: _lib.MVK_TYPE_I8}
_LAYOUTS = {"half": _lib.MVK_ROTARY_HALF, "interleaved": _lib.MVK_ROTARY_INTERLEAVED}
_SCALINGS = {None: _lib.MVK_SCALE_NONE, "linear": _lib.MVK_SCALE_LINEAR, "base": _lib.MVK_SCALE_BASE,
             "parts": _lib.MVK_SCALE_PARTS}

__all__ = ["FIELD", "KVCache", "Sequences", "rotary_table", "rotary", "rotary_append", "cache_read", "paged_attention",
           "cache_evict"]


def _rows(t: torch.Tensor, name: str, T: int, heads: int | None, dim: int):
    """T x heads x dim (heads None: any), any strides but a contiguous last axis."""
    # (plain comparisons: these checks cost as much as a launch if written with loops)
    kind = _TYPES.get(t.dtype) if isinstance(t, torch.Tensor) and t.is_cuda else None
    if kind is None:
        raise TypeError(f"{name} must be a CUDA tensor of bfloat16, float16, float32 or int32 (field)")
    shape = t.shape
    if len(shape) != 3 or shape[0] != T or shape[2] != dim or (heads is not None and shape[1] != heads):
        raise ValueError(f"{name} has shape {tuple(shape)}, expected (T, heads, dim) = {(T, heads, dim)}")
    a, b, c = t.stride()
    if c != 1 and dim > 1:
        raise ValueError(f"{name}: the last axis must be contiguous")
    return _lib.MvkRows(t.data_ptr(), kind, a, b)


@dataclass
class KVCache:
    """The pools of one layer: pages x kv_heads x page_size x dim each (views
    with other strides will do; the last axis is contiguous).  A cache held in 8
    bits (K and V float8_e4m3fn or int8) has k_exp and v_exp, pages x kv_heads x
    page_size int8 of any strides: an entry's row is codes * 2^exponent, what
    rotary_append rounds to and attention computes with, in bfloat16, exactly."""
    K: torch.Tensor
    V: torch.Tensor
    k_exp: torch.Tensor | None = None
    v_exp: torch.Tensor | None = None

    @classmethod
    def allocate(cls, pages: int, kv_heads: int, page_size: int, dim: int, dtype=torch.bfloat16,
                 device="cuda") -> "KVCache":
        shape = (pages, kv_heads, page_size)
        pools = [torch.zeros((*shape, dim), dtype=dtype, device=device) for _ in range(2)]
        if dtype in (torch.float8_e4m3fn, torch.int8):
            pools += [torch.zeros(shape, dtype=torch.int8, device=device) for _ in range(2)]
        return cls(*pools)

    @property
    def query_dtype(self):
        """Of the queries of paged_attention over this cache (bfloat16 where it is held in 8 bits)."""
        return torch.bfloat16 if self.k_exp is not None else self.K.dtype

    def struct(self):
        K, V = self.K, self.V
        if not (isinstance(K, torch.Tensor) and isinstance(V, torch.Tensor) and K.is_cuda and V.is_cuda):
            raise TypeError("K and V must be CUDA tensors")
        kind = _CACHE_TYPES.get(K.dtype)
        if K.dtype != V.dtype or kind is None:
            raise TypeError("K and V must both be bfloat16, float16, float32, float8_e4m3fn or int8, got "
                            f"{K.dtype}, {V.dtype}")
        shape = K.shape
        if len(shape) != 4 or shape != V.shape:
            raise ValueError(f"K and V must be pages x kv_heads x page_size x dim, got {tuple(shape)}, {tuple(V.shape)}")
        n, h, p, d = shape
        ka, kb, kc, kd = K.stride()
        va, vb, vc, vd = V.stride()
        if (kd != 1 or vd != 1) and d > 1:
            raise ValueError("K and V: the last axis must be contiguous")
        if kind != _lib.MVK_TYPE_E4M3 and kind != _lib.MVK_TYPE_I8:
            if self.k_exp is not None or self.v_exp is not None:
                raise ValueError("k_exp and v_exp belong to a cache held in 8 bits")
            return _lib.MvkKv(K.data_ptr(), V.data_ptr(), kind, n, h, p, d, ka, kb, kc, va, vb, vc)
        device, rows = K.get_device(), shape[:3]
        return _lib.MvkKv8(K.data_ptr(), V.data_ptr(), kind, n, h, p, d, ka, kb, kc, va, vb, vc,
                           _exps(self.k_exp, "k_exp", rows, device), _exps(self.v_exp, "v_exp", rows, device),
                           *self.k_exp.stride(), *self.v_exp.stride())


def _exps(x, name: str, shape, device: int):
    if not isinstance(x, torch.Tensor) or x.dtype != torch.int8 or x.get_device() != device:
        raise TypeError(f"{name} must be an int8 tensor on K's device (the cache is held in 8 bits)")
    if x.shape != shape:
        raise ValueError(f"{name} has shape {tuple(x.shape)}, expected {tuple(shape)}")
    return x.data_ptr()


@dataclass
class Sequences:
    """The sequences of a call: table (count x width int32 page numbers), lens
    (count, entries with the new ones), q_start (count + 1, where each one's new
    tokens begin; not needed for eviction).  max_new: an upper bound of the new
    tokens of one sequence (None: the call's token rows).  It chooses attention's
    kernel, not its result: give 1 for a batch of single tokens, which without it
    runs the form for chunks (32 sequences over 8000 entries: 238 us for 191)."""
    table: torch.Tensor
    lens: torch.Tensor
    q_start: torch.Tensor | None = None
    max_new: int | None = None

    def struct(self, rows: int):
        table, starts = self.table, self.q_start
        count, width = table.shape
        stride, one = table.stride()
        if not table.is_cuda or table.dtype != torch.int32 or (one != 1 and width > 1):
            raise ValueError("table must be a CUDA int32 tensor with contiguous rows")
        lens = _dev(self.lens, torch.int32, (count,), "lens")
        starts = _dev(starts, torch.int32, (count + 1,), "q_start") if starts is not None else None
        most = rows if self.max_new is None or self.max_new > rows else int(self.max_new)
        return _lib.MvkSeqs(table.data_ptr(), stride, count, width, lens, starts, _lib.count(most))


def rotary_table(rot: int, rows: int, base: float = 10000.0, scaling: str | None = None, factor: float = 1.0,
                 original_len: float = 0.0, slow: float = 1.0, fast: float = 32.0, out: torch.Tensor | None = None,
                 device="cuda", stream=None) -> torch.Tensor:
    """Cosines and sines of positions 0 .. rows - 1 (rows x rot float32: rot / 2
    cosines, rot / 2 sines).  scaling for long contexts: "linear" (positions
    divided by factor), "base" (the base raised), "parts" (by wavelength)."""
    if scaling not in _SCALINGS:
        raise ValueError(f"scaling must be one of {sorted(k for k in _SCALINGS if k)} or None")
    if out is None:
        out = torch.empty((rows, rot), dtype=torch.float32, device=device)
    _lib.check("mvk_rotary_table", _lib.load().mvk_rotary_table(
        rot, rows, base, _SCALINGS[scaling], factor, original_len, slow, fast,
        _dev(out, torch.float32, (rows, rot), "out"), _stream(stream)))
    return out


def _rotary_call(q, k, v, positions, table, cache, seqs, layout, field_scale, out, p, stream):
    if layout not in _LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(_LAYOUTS)}")
    x = q if q is not None else k
    T, _, dim = x.shape
    ref = ctypes.byref
    qs = ks = vs = os_ = cs = ss = None
    heads = 0
    if q is not None:
        heads = q.shape[1]
        qs, os_ = ref(_rows(q, "q", T, heads, dim)), ref(_rows(out, "out", T, heads, dim))
    if k is not None:
        kv = cache.struct()
        heads_kv, dim_kv = kv.kv_heads, kv.dim
        ks, vs = ref(_rows(k, "k", T, heads_kv, dim_kv)), ref(_rows(v, "v", T, heads_kv, dim_kv))
        cs, ss = ref(kv), ref(seqs.struct(T))
    if field_scale is None:
        if x.dtype == torch.int32:
            raise ValueError("field inputs need field_scale, the value of 1")
        field_scale = 0.0
    rows, rot = table.shape
    _lib.check("mvk_rotary_append", _lib.load(p).mvk_rotary_append(
        qs, ks, vs, _lib.count(T), heads, dim, rot, _LAYOUTS[layout], _dev(positions, torch.int32, (T,), "positions"),
        _dev(table, torch.float32, None, "table"), rows, field_scale, os_, cs, ss, _stream(stream)))


def rotary(q: torch.Tensor, positions: torch.Tensor, table: torch.Tensor, layout: str = "half",
           field_scale: float | None = None, out: torch.Tensor | None = None, out_dtype=torch.bfloat16, p: int = P,
           stream=None) -> torch.Tensor:
    """Rotary positions alone: the first table.shape[1] elements of every head of
    q (T x heads x dim; floats, or field elements times field_scale), by the
    table's rows positions[t].  layout "half" pairs elements i and i + rot / 2,
    "interleaved" 2i and 2i + 1.  out may be q."""
    if out is None:
        out = torch.empty(q.shape, dtype=out_dtype, device=q.device)
    _rotary_call(q, None, None, positions, table, None, None, layout, field_scale, out, p, stream)
    return out


def rotary_append(q: torch.Tensor | None, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor,
                  table: torch.Tensor, cache: KVCache, seqs: Sequences, layout: str = "half",
                  field_scale: float | None = None, out: torch.Tensor | None = None, p: int = P, stream=None):
    """Rotary positions on new tokens' q and k, and k, v into their places of the
    cache, in one launch.  q: T x heads x dim (or None), k, v: T x kv_heads x dim,
    one type.  Returns the rotated q in the cache's type (bfloat16 where that is
    held in 8 bits)."""
    if q is not None and out is None:
        out = torch.empty(q.shape, dtype=cache.query_dtype, device=q.device)
    _rotary_call(q, k, v, positions, table, cache, seqs, layout, field_scale, out, p, stream)
    return out


def cache_read(cache: KVCache, seqs: Sequences, tokens: int | None = None, dtype=torch.bfloat16,
               k_out: torch.Tensor | None = None, v_out: torch.Tensor | None = None, p: int = P, stream=None):
    """The new tokens' entries as the cache holds them, as rows: (k, v), T x
    kv_heads x dim of bfloat16, float16 or float32; T is `tokens`, or that of k_out and
    v_out (with one of them, only that one is read).  For whole sequences: q_start
    with their lengths summed up.  Rows of no sequence are left alone (zeros where
    the call allocates them)."""
    cs = cache.struct()
    if k_out is None and v_out is None:
        if tokens is None:
            raise ValueError("tokens is needed where neither k_out nor v_out is given")
        k_out, v_out = (torch.empty((tokens, cs.kv_heads, cs.dim), dtype=dtype, device=cache.K.device) for _ in range(2))
        with torch.cuda.stream(stream) if stream is not None else nullcontext():  # (where the rows are written)
            k_out.zero_(), v_out.zero_()
    T = (k_out if k_out is not None else v_out).shape[0]
    if tokens is not None and tokens != T:
        raise ValueError(f"the rows have {T} tokens, not {tokens}")
    ref = ctypes.byref
    hk, dim = cs.kv_heads, cs.dim
    ks = ref(_rows(k_out, "k_out", T, hk, dim)) if k_out is not None else None
    vs = ref(_rows(v_out, "v_out", T, hk, dim)) if v_out is not None else None
    _lib.check("mvk_cache_read", _lib.load(p).mvk_cache_read(ref(cs), ref(seqs.struct(T)), _lib.count(T), ks, vs,
                                                             _stream(stream)))
    return k_out, v_out


def paged_attention(q: torch.Tensor, cache: KVCache, seqs: Sequences, scale: float | None = None,
                    out: torch.Tensor | None = None, out_dtype=None, field_scale: float | None = None,
                    lse: torch.Tensor | None = None, weights: torch.Tensor | None = None,
                    weights_out: torch.Tensor | None = None, p: int = P, stream=None) -> torch.Tensor:
    """Attention of the new tokens q (T x heads x dim, already in the cache as
    keys and values) over their sequences' entries.  scale: dim ** -0.5 by
    default.  out_dtype: q's by default, float32, or FIELD: out / field_scale
    rounded into the field; out may be q where no weights are collected.  lse: T x heads float32, written.  weights,
    weights_out (count x kv_heads x width * page_size float32; may be one
    tensor): the attention weight every entry has collected, before and after
    (weights None with weights_out: from zero)."""
    T, heads, dim = q.shape
    if out is None:
        out = q.new_empty(q.shape) if out_dtype is None else torch.empty(q.shape, dtype=out_dtype, device=q.device)
    if out.dtype == torch.int32 and field_scale is None:
        raise ValueError("field outputs need field_scale, the value of 1")
    cs, ss = cache.struct(), seqs.struct(T)
    qs, os_ = _rows(q, "q", T, None, cs.dim), _rows(out, "out", T, heads, dim)
    w_in = w_out = None
    w_seq = w_head = 0
    if weights is not None and weights_out is None:
        weights_out = weights
    if weights_out is not None:
        w_out, w_seq, w_head = _weights(weights_out, ss, cs, "weights_out")
        if weights is not None:
            w_in, a, b = _weights(weights, ss, cs, "weights")
            if (a, b) != (w_seq, w_head):
                raise ValueError("weights and weights_out must have the same strides")
    ref = ctypes.byref
    _lib.check("mvk_paged_attention", _lib.load(p).mvk_paged_attention(
        ref(qs), _lib.count(T), heads, ref(cs), ref(ss), dim**-0.5 if scale is None else scale, ref(os_),
        field_scale or 0.0,
        _dev(lse, torch.float32, (T, heads), "lse") if lse is not None else None, w_in, w_out, w_seq, w_head,
        _stream(stream)))
    return out


def _weights(w: torch.Tensor, ss, cs, name: str):
    if not isinstance(w, torch.Tensor) or not w.is_cuda or w.dtype != torch.float32:
        raise TypeError(f"{name} must be a CUDA float32 tensor")
    if w.dim() != 3 or w.shape[0] != ss.count or w.shape[1] != cs.kv_heads or w.shape[2] < ss.width * cs.page_size:
        raise ValueError(f"{name} has shape {tuple(w.shape)}, expected {(ss.count, cs.kv_heads)} x at least "
                         f"{ss.width * cs.page_size}")
    a, b, c = w.stride()
    if c != 1:
        raise ValueError(f"{name}: the last axis must be contiguous")
    return w.data_ptr(), a, b


def cache_evict(cache: KVCache, seqs: Sequences, weights: torch.Tensor, dst: KVCache, dst_table: torch.Tensor,
                budget: int, recent: int = 0, sinks: int = 0, weights_out: torch.Tensor | None = None,
                kept: torch.Tensor | None = None, lens_out: torch.Tensor | None = None, stream=None):
    """Keep at most `budget` entries of every sequence and kv head: the first
    `sinks`, the last `recent` and the heaviest others by `weights` (count x
    kv_heads x width * page_size), copied in order into dst_table's pages of dst,
    their weights into weights_out (in no memory of weights).  Returns (kept,
    lens): the kept entries' indices (count x kv_heads x budget, -1 beyond) and
    how many each sequence has now (lens_out, which may be seqs.lens)."""
    cs, ds, ss = cache.struct(), dst.struct(), seqs.struct(0)
    dev = weights.device
    if kept is None:
        kept = torch.empty((ss.count, cs.kv_heads, budget), dtype=torch.int32, device=dev)
    if lens_out is None:
        lens_out = torch.empty((ss.count,), dtype=torch.int32, device=dev)
    w, w_seq, w_head = _weights(weights, ss, cs, "weights")
    wo = o_seq = o_head = 0
    if weights_out is not None:
        if (not weights_out.is_cuda or weights_out.dtype != torch.float32 or weights_out.dim() != 3
                or weights_out.shape[:2] != (ss.count, cs.kv_heads) or weights_out.stride(2) != 1
                or weights_out.shape[2] < min(budget, ss.width * cs.page_size)):
            raise ValueError("weights_out must be a CUDA float32 tensor, count x kv_heads x at least budget")
        wo, (o_seq, o_head, _) = weights_out.data_ptr(), weights_out.stride()
    if (not dst_table.is_cuda or dst_table.dtype != torch.int32 or dst_table.dim() != 2
            or dst_table.shape[0] != ss.count or (dst_table.shape[1] > 1 and dst_table.stride(1) != 1)):
        raise ValueError("dst_table must be a CUDA int32 tensor, count x pages, with contiguous rows")
    ref = ctypes.byref
    _lib.check("mvk_cache_evict", _lib.load().mvk_cache_evict(
        ref(cs), ref(ss), w, w_seq, w_head, budget, recent, sinks, ref(ds), dst_table.data_ptr(),
        dst_table.stride(0), dst_table.shape[1], wo or None, o_seq, o_head,
        _dev(kept, torch.int32, (ss.count, cs.kv_heads, budget), "kept"),
        _dev(lens_out, torch.int32, (ss.count,), "lens_out"), _stream(stream)))
    return kept, lens_out
