"""Binding of the paged key/value cache (include/spmm_cache.h): argument marshalling and checks of tensors.

Functions have the names of their C declarations.  Device operands are torch tensors, whose types, layouts and sizes are
checked here, or raw integer addresses, which are not; sizes that a tensor's shape says are taken from it.  What is as it
should be is marshalled in C (csrc_cache/native_cache.c, which takes the place of the functions here at the end of this
file and hands everything else back to them).
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
from typing import Optional

from .binding import OUT_TYPES, SPMM_OUT_F32, SPMM_OUT_S8, SPMM_OUT_U8, _check, _nbytes, lib

__all__ = [
    "SPMM_CACHE_BF16", "SPMM_CACHE_S8", "SPMM_OUT_BF16", "CACHE_EXPORTS", "spmm_cache_t", "spmm_batch_t", "spmm_append_t", "spmm_attend_t",
    "make_cache", "make_batch", "make_append", "make_attend", "make_rope", "spmm_cache_append", "spmm_cache_attend", "spmm_attend_work_bytes",
    "spmm_cache_fork", "spmm_cache_compact", "spmm_cache_copy", "spmm_cache_work_bytes",
    "spmm_select_t", "spmm_weigh_t", "spmm_evict_t", "make_select", "make_weigh", "make_evict", "spmm_cache_bounds", "spmm_cache_score", "spmm_cache_select",
    "spmm_selected_work_bytes", "spmm_cache_attend_selected", "spmm_weigh_work_bytes", "spmm_cache_weigh", "spmm_cache_evict",
]

SPMM_CACHE_BF16, SPMM_CACHE_S8 = 0, 1
SPMM_OUT_BF16 = 4
ATTEND_OUT_TYPES = {"f32": SPMM_OUT_F32, "bf16": SPMM_OUT_BF16, "s8": SPMM_OUT_S8, "u8": SPMM_OUT_U8}
_OUT_BYTES = {SPMM_OUT_F32: 4, SPMM_OUT_BF16: 2, SPMM_OUT_S8: 1, SPMM_OUT_U8: 1}

CACHE_EXPORTS = ("spmm_cache_append", "spmm_cache_attend", "spmm_attend_work_bytes", "spmm_cache_fork", "spmm_cache_compact",
                 "spmm_cache_copy", "spmm_cache_work_bytes", "spmm_cache_bounds", "spmm_cache_score", "spmm_cache_select", "spmm_selected_work_bytes",
                 "spmm_cache_attend_selected", "spmm_weigh_work_bytes", "spmm_cache_weigh", "spmm_cache_evict")

_i64, _i32, _vp, _f32 = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_float


class spmm_cache_t(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp), ("type", ctypes.c_int), ("n_layers", _i32), ("n_heads", _i32),
                ("head_dim", _i32), ("page_tokens", _i32), ("n_pages", _i64), ("bounds", _vp), ("weight", _vp)]


class spmm_batch_t(ctypes.Structure):
    _fields_ = [("n_seqs", _i64), ("q_start", _vp), ("kv_len", _vp), ("table", _vp), ("ld_table", _i64)]


class spmm_append_t(ctypes.Structure):
    _fields_ = [("q_heads", _i32), ("x_type", ctypes.c_int), ("x_scale", _f32), ("x_zero_point", _i32), ("q_weight", _vp), ("k_weight", _vp),
                ("eps", _f32), ("rope", _vp), ("rope_len", _i64), ("rope_dim", _i32), ("interleaved", _i32), ("positions", _vp)]


class spmm_attend_t(ctypes.Structure):
    _fields_ = [("q_heads", _i32), ("max_new", _i64), ("scale", _f32), ("causal", _i32), ("window", _i32), ("out_type", _i32),
                ("out_scale", _f32), ("out_zero_point", _i32)]


class spmm_select_t(ctypes.Structure):
    _fields_ = [("q_heads", _i32), ("pages", _i32), ("first", _i32), ("last", _i32), ("causal", _i32), ("window", _i32)]


class spmm_weigh_t(ctypes.Structure):
    _fields_ = [("q_heads", _i32), ("max_new", _i64), ("scale", _f32), ("causal", _i32), ("window", _i32), ("decay", _f32)]


class spmm_evict_t(ctypes.Structure):
    _fields_ = [("first", _i32), ("recent", _i32), ("most", _i64)]


_bound = _native = None


def _functions() -> ctypes.CDLL:
    """The library, its functions of the cache declared."""
    global _bound
    if _bound is None:
        L = lib()
        cache, batch = ctypes.POINTER(spmm_cache_t), ctypes.POINTER(spmm_batch_t)
        for name, args in (
                ("spmm_cache_append", [cache, _i32, batch, _vp, _i64, _i64, ctypes.POINTER(spmm_append_t), _vp, _vp]),
                ("spmm_cache_attend", [cache, _i32, batch, _vp, _i64, ctypes.POINTER(spmm_attend_t), _vp, _i64, _vp, _vp]),
                ("spmm_attend_work_bytes", [cache, _i64, _i64, ctypes.POINTER(spmm_attend_t), ctypes.POINTER(_i64)]),
                ("spmm_cache_fork", [cache, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _vp, _vp]),
                ("spmm_cache_compact", [cache, _vp, _i64, _i64, _vp, _vp, _vp, _vp]),
                ("spmm_cache_copy", [cache, _vp, _vp, _i64, _vp]),
                ("spmm_cache_work_bytes", [cache, _i64, ctypes.POINTER(_i64)]),
                ("spmm_cache_bounds", [cache, _i32, batch, _i64, _vp]),
                ("spmm_cache_score", [cache, _i32, batch, _vp, _i64, ctypes.POINTER(spmm_select_t), _vp, _i64, _vp]),
                ("spmm_cache_select", [cache, batch, _vp, _i64, _i64, ctypes.POINTER(spmm_select_t), _vp, _vp]),
                ("spmm_selected_work_bytes", [cache, _i64, ctypes.POINTER(spmm_attend_t), _i64, ctypes.POINTER(_i64)]),
                ("spmm_cache_attend_selected", [cache, _i32, batch, _vp, _i64, ctypes.POINTER(spmm_attend_t), _vp, _i64, _vp, _i64, _vp, _vp]),
                ("spmm_weigh_work_bytes", [cache, batch, _i64, ctypes.POINTER(spmm_weigh_t), ctypes.POINTER(_i64)]),
                ("spmm_cache_weigh", [cache, _i32, batch, _vp, _i64, ctypes.POINTER(spmm_weigh_t), _vp, _vp]),
                ("spmm_cache_evict", [cache, _vp, _i64, _vp, _i64, _vp, ctypes.POINTER(spmm_evict_t), _vp, _vp, _vp, _vp])):
            f = getattr(L, name)
            f.restype, f.argtypes = ctypes.c_int, args
        if _native is not None:
            _native.bind(*(ctypes.cast(getattr(L, n), ctypes.c_void_p).value for n in (
                "spmm_cache_append", "spmm_cache_attend", "spmm_attend_work_bytes", "spmm_cache_fork", "spmm_cache_compact", "spmm_cache_work_bytes",
                "spmm_cache_bounds", "spmm_cache_score", "spmm_cache_select", "spmm_selected_work_bytes", "spmm_cache_attend_selected",
                "spmm_weigh_work_bytes", "spmm_cache_weigh", "spmm_cache_evict")))
        _bound = L
    return _bound


def _struct(v, kind):
    """A description as a ctypes structure (those made in C hold the same bytes)."""
    return v if isinstance(v, kind) else kind.from_buffer_copy(v)


def _name(t) -> str:
    return str(t.dtype).rsplit(".", 1)[-1]


def _tensor(t, what: str, dtype: str, shape=None, need: Optional[int] = None):
    """The address of a device operand; a tensor must be contiguous, of this type, and of this shape or of at least `need` elements."""
    if t is None or isinstance(t, int):
        return t
    if _name(t) != dtype or not t.is_contiguous() or (shape is not None and tuple(t.shape) != tuple(shape)) or (need is not None and t.numel() < need):
        raise ValueError("%s: a contiguous %s tensor%s is wanted, not %s of %s" % (
            what, dtype, " of shape %s" % (tuple(shape),) if shape is not None else " of %d elements" % need if need is not None else "", _name(t), tuple(t.shape)))
    return _address(t, what)


def _address(t, what: str):
    if not t.is_cuda:
        raise ValueError("%s: a tensor on the device is wanted" % what)
    return t.data_ptr()


def make_cache(k, v, k_scale=None, v_scale=None, bounds=None, weight=None) -> spmm_cache_t:
    """A cache over the caller's tensors: k [layers, pages, heads, page_tokens, head_dim], v [layers, pages, heads, head_dim, page_tokens],
    bfloat16, or int8 with scales [layers, pages, heads, page_tokens] in float32; for long contexts the keys' bounds
    [layers, pages, heads, 2, head_dim] in bfloat16 and the tokens' weights [layers, pages, heads, page_tokens] in float32."""
    layers, pages, heads, tokens, dim = k.shape
    kind = _name(k)
    if kind not in ("bfloat16", "int8"):
        raise ValueError("make_cache: keys in bfloat16 or int8 are wanted, not %s" % kind)
    if (kind == "int8") != (k_scale is not None) or (kind == "int8") != (v_scale is not None):
        raise ValueError("make_cache: int8 caches have scales, others have none")
    scales = (layers, pages, heads, tokens)
    c = spmm_cache_t(_tensor(k, "k", kind), _tensor(v, "v", kind, (layers, pages, heads, dim, tokens)), _tensor(k_scale, "k_scale", "float32", scales),
                     _tensor(v_scale, "v_scale", "float32", scales), SPMM_CACHE_S8 if kind == "int8" else SPMM_CACHE_BF16, layers, heads, dim, tokens, pages,
                     _tensor(bounds, "bounds", "bfloat16", (layers, pages, heads, 2, dim)), _tensor(weight, "weight", "float32", scales))
    c._keepalive = (k, v, k_scale, v_scale, bounds, weight)
    return c


def make_batch(q_start, kv_len, table) -> spmm_batch_t:
    """Sequences, their new tokens' columns, lengths and pages: int32 tensors [n_seqs + 1], [n_seqs], [n_seqs, width]."""
    n, width = table.shape
    b = spmm_batch_t(n, _tensor(q_start, "q_start", "int32", (n + 1,)), _tensor(kv_len, "kv_len", "int32", (n,)), _tensor(table, "table", "int32"), width)
    b._keepalive = (q_start, kv_len, table)
    return b


def make_rope(positions: int, dim: int, base: float = 10000.0):
    """Rotation table [positions, dim / 2, 2] of (cos, sin), angle i of position p being p * base^(-2 i / dim): host tensor, float32."""
    import torch
    turn = torch.arange(positions, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
    return torch.stack((turn.cos(), turn.sin()), dim=-1).float()


def make_append(q_heads: int, x_type="f32", x_scale: float = 1.0, x_zero_point: int = 0, q_weight=None, k_weight=None, eps: float = 1e-6,
                rope=None, interleaved=False, positions=None) -> spmm_append_t:
    """How queries, keys and values are made; rope: a tensor [positions, rope_dim / 2, 2] of (cos, sin)."""
    length, half = (0, 0) if rope is None else (rope.shape[0], rope.shape[1])
    a = spmm_append_t(q_heads, OUT_TYPES[x_type] if isinstance(x_type, str) else x_type, x_scale, x_zero_point, _tensor(q_weight, "q_weight", "float32"),
                      _tensor(k_weight, "k_weight", "float32"), eps, _tensor(rope, "rope", "float32", (length, half, 2)), length, 2 * half,
                      bool(interleaved), _tensor(positions, "positions", "int32"))
    a._keepalive = (q_weight, k_weight, rope, positions)
    return a


def make_attend(q_heads: int, max_new: int, scale: float, causal: bool = True, window: int = 0, out_type="bf16", out_scale: float = 1.0,
                out_zero_point: int = 0) -> spmm_attend_t:
    return spmm_attend_t(q_heads, max_new, scale, bool(causal), window, ATTEND_OUT_TYPES[out_type] if isinstance(out_type, str) else out_type,
                         out_scale, out_zero_point)


_X_TYPES = {SPMM_OUT_F32: "float32", SPMM_OUT_S8: "int8", SPMM_OUT_U8: "uint8"}
_O_TYPES = {SPMM_OUT_F32: "float32", SPMM_OUT_BF16: "bfloat16", SPMM_OUT_S8: "int8", SPMM_OUT_U8: "uint8"}


def _matrix(t, what: str, dtype: Optional[str], rows: int, cols: int, ld: int):
    """The address of a matrix of `rows` rows of pitch `ld`; a tensor must have the type and cover it."""
    if t is None or isinstance(t, int):
        return t
    if _name(t) != dtype:
        raise ValueError("%s: a %s tensor is wanted, not %s" % (what, dtype, _name(t)))
    if rows > 0 and cols > 0 and _nbytes(t) < ((rows - 1) * ld + cols) * t.element_size():
        raise ValueError("%s holds %d bytes behind its data pointer, the call touches %d" % (what, _nbytes(t), ((rows - 1) * ld + cols) * t.element_size()))
    return _address(t, what)


def spmm_cache_append(cache: spmm_cache_t, layer: int, batch: spmm_batch_t, x, T: int, ldx: int, how: spmm_append_t, q, stream=None) -> None:
    """New tokens' queries to q, their keys and values to the cache; asynchronous on `stream` (a raw hipStream_t value, None = default stream)."""
    keep = getattr(how, "_keepalive", (None,) * 4)
    cache, batch, how = _struct(cache, spmm_cache_t), _struct(batch, spmm_batch_t), _struct(how, spmm_append_t)
    rows = (how.q_heads + 2 * cache.n_heads) * cache.head_dim
    for w in keep[:2]:
        _tensor(w, "weight", "float32", need=cache.head_dim)
    if keep[3] is not None:
        _tensor(keep[3], "positions", "int32", need=T)
    _check(_functions().spmm_cache_append(cache, layer, batch, _matrix(x, "x", _X_TYPES.get(how.x_type), rows, T, ldx), T, ldx, how,
                                          _tensor(q, "q", "bfloat16", need=T * how.q_heads * cache.head_dim), stream), "spmm_cache_append")


def spmm_attend_work_bytes(cache: spmm_cache_t, n_seqs: int, T: int, how: spmm_attend_t) -> int:
    n = _i64()
    cache, how = _struct(cache, spmm_cache_t), _struct(how, spmm_attend_t)
    _check(_functions().spmm_attend_work_bytes(cache, n_seqs, T, how, n), "spmm_attend_work_bytes")
    return n.value


def spmm_cache_attend(cache: spmm_cache_t, layer: int, batch: spmm_batch_t, q, T: int, how: spmm_attend_t, out, ldo: int, work, stream=None) -> None:
    """out [q_heads * head_dim][ldo] = attention of the new tokens; work: a tensor of spmm_attend_work_bytes bytes."""
    cache, batch, how = _struct(cache, spmm_cache_t), _struct(batch, spmm_batch_t), _struct(how, spmm_attend_t)
    values = how.q_heads * cache.head_dim
    if work is not None and not isinstance(work, int) and _nbytes(work) < _in_python["spmm_attend_work_bytes"](cache, batch.n_seqs, T, how):
        raise ValueError("work holds %d bytes, %d are wanted" % (_nbytes(work), _in_python["spmm_attend_work_bytes"](cache, batch.n_seqs, T, how)))
    _check(_functions().spmm_cache_attend(cache, layer, batch, _tensor(q, "q", "bfloat16", need=T * values), T, how,
                                          _matrix(out, "out", _O_TYPES.get(how.out_type), values, T, ldo), ldo, work if work is None or isinstance(work, int) else _address(work, "work"), stream), "spmm_cache_attend")


def spmm_cache_work_bytes(cache: spmm_cache_t, n_rows: int) -> int:
    n = _i64()
    cache = _struct(cache, spmm_cache_t)
    _check(_functions().spmm_cache_work_bytes(cache, n_rows, n), "spmm_cache_work_bytes")
    return n.value


def _page_work(cache, n_rows, work):
    if work is not None and not isinstance(work, int) and _nbytes(work) < _in_python["spmm_cache_work_bytes"](cache, n_rows):
        raise ValueError("work holds %d bytes, %d are wanted" % (_nbytes(work), _in_python["spmm_cache_work_bytes"](cache, n_rows)))
    return work if work is None or isinstance(work, int) else _address(work, "work")


def spmm_cache_fork(cache: spmm_cache_t, table, kv_len, parent, keep, want, table_out, kv_len_out, info, work, stream=None) -> None:
    """The next generation of the sequences: int32 tensors table [rows, width], kv_len [rows] -> table_out [new rows, width], kv_len_out;
    parent, keep, want [new rows]; info [4]; work: spmm_cache_work_bytes bytes."""
    cache = _struct(cache, spmm_cache_t)
    (rows_in, width), rows = table.shape, table_out.shape[0]
    i = "int32"
    _check(_functions().spmm_cache_fork(
        cache, _tensor(table, "table", i), width, _tensor(kv_len, "kv_len", i, (rows_in,)), rows_in, _tensor(parent, "parent", i, (rows,)),
        _tensor(keep, "keep", i, (rows,)), _tensor(want, "want", i, (rows,)), rows, _tensor(table_out, "table_out", i, (rows, width)),
        _tensor(kv_len_out, "kv_len_out", i, (rows,)), _tensor(info, "info", i, need=4), _page_work(cache, rows, work), stream), "spmm_cache_fork")


def spmm_cache_compact(cache: spmm_cache_t, table, table_out, info, work, stream=None) -> None:
    """Pages in use to the front of the pool; table_out (which may be table) takes the new numbers."""
    cache = _struct(cache, spmm_cache_t)
    rows, width = table.shape
    _check(_functions().spmm_cache_compact(cache, _tensor(table, "table", "int32"), width, rows, _tensor(table_out, "table_out", "int32", (rows, width)),
                                           _tensor(info, "info", "int32", need=4), _page_work(cache, rows, work), stream), "spmm_cache_compact")


def spmm_cache_copy(cache: spmm_cache_t, src, dst, n: int, stream=None) -> None:
    """Pages src[i] to dst[i] in all layers, i < n (int32 tensors)."""
    cache = _struct(cache, spmm_cache_t)
    _check(_functions().spmm_cache_copy(cache, _tensor(src, "src", "int32", need=n), _tensor(dst, "dst", "int32", need=n), n, stream), "spmm_cache_copy")


def make_select(q_heads: int, pages: int, first: int = 1, last: int = 1, causal: bool = True, window: int = 0) -> spmm_select_t:
    """Lists of at most `pages` pages, the first `first` and the last `last` visible ones among them."""
    return spmm_select_t(q_heads, pages, first, last, bool(causal), window)


def make_weigh(q_heads: int, max_new: int, scale: float, causal: bool = True, window: int = 0, decay: float = 1.0) -> spmm_weigh_t:
    """The last max_new new tokens of a sequence count; what earlier calls added up is multiplied by decay."""
    return spmm_weigh_t(q_heads, max_new, scale, bool(causal), window, decay)


def make_evict(first: int, recent: int, most: int) -> spmm_evict_t:
    """The first and the most recent tokens stay, and at most `most` of a row in all."""
    return spmm_evict_t(first, recent, most)


def _scratch(work, need: int):
    if work is not None and not isinstance(work, int) and _nbytes(work) < need:
        raise ValueError("work holds %d bytes, %d are wanted" % (_nbytes(work), need))
    return work if work is None or isinstance(work, int) else _address(work, "work")


def spmm_cache_bounds(cache: spmm_cache_t, layer: int, batch: spmm_batch_t, T: int, stream=None) -> None:
    """Bounds of the keys of the pages that the batch's new tokens lie in."""
    cache, batch = _struct(cache, spmm_cache_t), _struct(batch, spmm_batch_t)
    _check(_functions().spmm_cache_bounds(cache, layer, batch, T, stream), "spmm_cache_bounds")


def spmm_cache_score(cache: spmm_cache_t, layer: int, batch: spmm_batch_t, q, T: int, how: spmm_select_t, scores, lds: int, stream=None) -> None:
    """scores [T][n_heads][lds] (float32) = upper bounds of the new tokens' products with the keys of each page."""
    cache, batch, how = _struct(cache, spmm_cache_t), _struct(batch, spmm_batch_t), _struct(how, spmm_select_t)
    _check(_functions().spmm_cache_score(cache, layer, batch, _tensor(q, "q", "bfloat16", need=T * how.q_heads * cache.head_dim), T, how,
                                         _tensor(scores, "scores", "float32", need=T * cache.n_heads * lds), lds, stream), "spmm_cache_score")


def spmm_cache_select(cache: spmm_cache_t, batch: spmm_batch_t, scores, T: int, lds: int, how: spmm_select_t, lists, stream=None) -> None:
    """lists [T][n_heads][pages] (int32) = the pages that each new token reads, of scores [T][n_heads][lds]."""
    cache, batch, how = _struct(cache, spmm_cache_t), _struct(batch, spmm_batch_t), _struct(how, spmm_select_t)
    _check(_functions().spmm_cache_select(cache, batch, _tensor(scores, "scores", "float32", need=T * cache.n_heads * lds), T, lds, how,
                                          _tensor(lists, "lists", "int32", need=T * cache.n_heads * how.pages), stream), "spmm_cache_select")


def spmm_selected_work_bytes(cache: spmm_cache_t, T: int, how: spmm_attend_t, pages: int) -> int:
    n = _i64()
    cache, how = _struct(cache, spmm_cache_t), _struct(how, spmm_attend_t)
    _check(_functions().spmm_selected_work_bytes(cache, T, how, pages, n), "spmm_selected_work_bytes")
    return n.value


def spmm_cache_attend_selected(cache: spmm_cache_t, layer: int, batch: spmm_batch_t, q, T: int, how: spmm_attend_t, lists, pages: int, out, ldo: int, work, stream=None) -> None:
    """spmm_cache_attend over the pages of lists [T][n_heads][pages] (int32); work: a tensor of spmm_selected_work_bytes bytes."""
    cache, batch, how = _struct(cache, spmm_cache_t), _struct(batch, spmm_batch_t), _struct(how, spmm_attend_t)
    values = how.q_heads * cache.head_dim
    need = 0 if work is None or isinstance(work, int) else _in_python["spmm_selected_work_bytes"](cache, T, how, pages)
    _check(_functions().spmm_cache_attend_selected(
        cache, layer, batch, _tensor(q, "q", "bfloat16", need=T * values), T, how, _tensor(lists, "lists", "int32", need=T * cache.n_heads * pages), pages,
        _matrix(out, "out", _O_TYPES.get(how.out_type), values, T, ldo), ldo, _scratch(work, need), stream), "spmm_cache_attend_selected")


def spmm_weigh_work_bytes(cache: spmm_cache_t, batch: spmm_batch_t, T: int, how: spmm_weigh_t) -> int:
    n = _i64()
    cache, batch, how = _struct(cache, spmm_cache_t), _struct(batch, spmm_batch_t), _struct(how, spmm_weigh_t)
    _check(_functions().spmm_weigh_work_bytes(cache, batch, T, how, n), "spmm_weigh_work_bytes")
    return n.value


def spmm_cache_weigh(cache: spmm_cache_t, layer: int, batch: spmm_batch_t, q, T: int, how: spmm_weigh_t, work, stream=None) -> None:
    """The new tokens' attention added to the cache's weights; work: a tensor of spmm_weigh_work_bytes bytes."""
    cache, batch, how = _struct(cache, spmm_cache_t), _struct(batch, spmm_batch_t), _struct(how, spmm_weigh_t)
    need = 0 if work is None or isinstance(work, int) else _in_python["spmm_weigh_work_bytes"](cache, batch, T, how)
    _check(_functions().spmm_cache_weigh(cache, layer, batch, _tensor(q, "q", "bfloat16", need=T * how.q_heads * cache.head_dim), T, how,
                                         _scratch(work, need), stream), "spmm_cache_weigh")


def spmm_cache_evict(cache: spmm_cache_t, table, kv_len, keep, how: spmm_evict_t, table_to, kv_len_out, kept, stream=None) -> None:
    """What stays of each row of table [rows, width] goes to the front of the row of table_to (which may be table); int32 tensors kv_len, keep,
    kv_len_out [rows], kept [layers, rows, n_heads, how.most]."""
    cache, how = _struct(cache, spmm_cache_t), _struct(how, spmm_evict_t)
    rows, width = table.shape
    i = "int32"
    _check(_functions().spmm_cache_evict(
        cache, _tensor(table, "table", i), width, _tensor(kv_len, "kv_len", i, (rows,)), rows, _tensor(keep, "keep", i, (rows,)), how,
        _tensor(table_to, "table_to", i, (rows, width)), _tensor(kv_len_out, "kv_len_out", i, (rows,)),
        _tensor(kept, "kept", i, need=cache.n_layers * rows * cache.n_heads * how.most), stream), "spmm_cache_evict")


_FAST = ("make_cache", "make_batch", "make_append", "make_attend", "spmm_cache_append", "spmm_cache_attend", "spmm_attend_work_bytes", "spmm_cache_fork",
         "spmm_cache_compact", "spmm_cache_work_bytes", "make_select", "make_weigh", "make_evict", "spmm_cache_bounds", "spmm_cache_score", "spmm_cache_select",
         "spmm_selected_work_bytes", "spmm_cache_attend_selected", "spmm_weigh_work_bytes", "spmm_cache_weigh", "spmm_cache_evict")
NATIVE_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_native_cache.so")
_in_python = {n: globals()[n] for n in _FAST}       # (the tests of the checks call these too)

if os.path.exists(NATIVE_PATH):
    _spec = importlib.util.spec_from_file_location(__package__ + "._native_cache", NATIVE_PATH)
    _native = importlib.util.module_from_spec(_spec)
    _spec.loader.exec_module(_native)
    _native.hooks(_check, *_in_python.values())
    globals().update({n: getattr(_native, n) for n in _FAST})
