"""Operators of a decode step, over memory 4 bits wide and over a paged cache in bf16 or fp32: the ctypes binding of ``include/rsd_ops.h``.

Device buffers are torch tensors; every call goes to torch's current stream and returns without waiting.  Outputs and
workspaces come from torch's allocator, so they follow its rules for streams and graphs.  A wrong argument raises
:class:`~.binding.RsdError` before anything is enqueued.

* ``rsd_w4_pack`` / ``rsd_w4_linear``: weights in 4 bits, and products with them.
* ``rsd_kv4_cache``: an empty paged 4-bit cache.  A cache is any tuple ``(pool, table, kv_len)``: pages ``[n_pages, n_kv_heads, 17 *
  head_dim]`` uint8, page numbers ``[batch, max_pages]`` int32 (-1: none), entries of each sequence ``[batch]`` int32.
* ``rsd_kv4_append`` / ``rsd_kv4_read``: entries in and out.
* ``rsd_kv4_attention``: attention over the cache, with the weight every entry received on request.
* ``rsd_kv4_evict``: cuts each sequence back to a budget of entries by that weight.
* ``rsd_rope``: a rotation by position, its frequencies scaled for long contexts if wanted.  ``rsd_qk_rope``: norms of the heads of queries and keys, and that
  rotation, in one pass.
* ``rsd_kv_cache``: an empty paged cache in bf16 or fp32.  A cache is any tuple ``(pool, table, kv_len)``: pages ``[n_pages, n_kv_heads, 2, 16 * head_dim]``, the rest as
  above.
* ``rsd_kv_append`` / ``rsd_kv_read``: entries in, keys normed and rotated on the way, and out.
* ``rsd_kv_attention``: attention over the cache, with a sliding window and first tokens that stay visible if wanted.

The formats and the layouts are described in the header.
"""
from __future__ import annotations

import ctypes as C
import math
import struct
from functools import lru_cache
from operator import index
from typing import NamedTuple, Optional, Tuple

import torch

from . import binding as _b

__all__ = ["W4", "Kv4Cache", "rsd_w4_pack", "rsd_w4_linear", "rsd_kv4_cache", "rsd_kv4_append", "rsd_kv4_read", "rsd_kv4_attention",
           "rsd_kv4_evict", "Rope", "KvCache", "rsd_rope", "rsd_qk_rope", "rsd_kv_cache", "rsd_kv_append", "rsd_kv_read", "rsd_kv_attention", "OPS_EXPORTED_SYMBOLS"]

OPS_EXPORTED_SYMBOLS = ["rsd_op_last_error", "rsd_w4_pack", "rsd_w4_linear_workspace", "rsd_w4_linear", "rsd_kv4_append", "rsd_kv4_read",
                        "rsd_kv4_attention_workspace", "rsd_kv4_attention", "rsd_kv4_evict_workspace", "rsd_kv4_evict", "rsd_rope_frequencies",
                        "rsd_qk_rope", "rsd_kv_append", "rsd_kv_read", "rsd_kv_attention_workspace", "rsd_kv_attention"]

PAGE = 16
_TYPE = {torch.float32: 0, torch.bfloat16: 1}
_i32, _u8, _f32 = torch.int32, torch.uint8, torch.float32


class W4(NamedTuple):
    """A weight matrix ``[n, k]`` in 4-bit tiles."""
    codes: torch.Tensor
    scales: torch.Tensor
    n: int
    k: int


class Kv4Cache(NamedTuple):
    pool: torch.Tensor
    table: torch.Tensor
    kv_len: torch.Tensor


class Rope(NamedTuple):
    """A rotation: radians per position of every pair (float64 ``[rot_dim / 2]``), pairs (2 i, 2 i + 1) or (i, i + rot_dim / 2), what the result is multiplied by."""
    freq: torch.Tensor
    interleaved: bool
    magnitude: float


class KvCache(NamedTuple):
    pool: torch.Tensor
    table: torch.Tensor
    kv_len: torch.Tensor


class _W4(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("n", C.c_int32), ("k", C.c_int32)]


class _Cache(C.Structure):
    _fields_ = [("pool", C.c_void_p), ("table", C.c_void_p), ("kv_len", C.c_void_p), ("n_pages", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("batch", C.c_int32), ("max_pages", C.c_int32)]


class _Book(C.Structure):
    _fields_ = [("scores", C.c_void_p), ("positions", C.c_void_p), ("score_b", C.c_int64), ("score_h", C.c_int64),
                ("position_b", C.c_int64), ("position_h", C.c_int64)]


class _Attn(C.Structure):
    _fields_ = [("q", C.c_void_p), ("out", C.c_void_p), ("lse", C.c_void_p), ("q_row", C.c_int64), ("q_head", C.c_int64),
                ("out_row", C.c_int64), ("out_head", C.c_int64), ("row_start", C.c_void_p), ("rows", C.c_int32),
                ("max_rows", C.c_int32), ("n_heads", C.c_int32), ("max_kv", C.c_int32), ("dtype", C.c_int32), ("scale", C.c_float)]


class _Rope(C.Structure):
    _fields_ = [("freq", C.c_void_p), ("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("magnitude", C.c_float)]


class _Heads(C.Structure):
    _fields_ = [("x", C.c_void_p), ("out", C.c_void_p), ("weight", C.c_void_p), ("row", C.c_int64), ("head", C.c_int64), ("out_row", C.c_int64),
                ("out_head", C.c_int64), ("n_heads", C.c_int32)]


class _KvCache(C.Structure):
    _fields_ = [*_Cache._fields_, ("dtype", C.c_int32)]


class _KvAttn(C.Structure):
    _fields_ = [("q", C.c_void_p), ("out", C.c_void_p), ("lse", C.c_void_p), ("q_row", C.c_int64), ("q_head", C.c_int64),
                ("out_row", C.c_int64), ("out_head", C.c_int64), ("row_start", C.c_void_p), ("rows", C.c_int32), ("max_rows", C.c_int32), ("n_heads", C.c_int32),
                ("max_kv", C.c_int32), ("window", C.c_int32), ("sinks", C.c_int32), ("dtype", C.c_int32), ("scale", C.c_float)]


_lib = None


def _load():
    """The library with the argument types of its operators set."""
    global _lib
    lib = _b.load_library()
    p, i32, i64, u64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64
    lib.rsd_op_last_error.restype = C.c_char_p
    lib.rsd_w4_pack.argtypes = [p, i32, i64, i32, i32, p, p, p]
    lib.rsd_w4_linear.argtypes = [p, p, i64, p, i64, i32, i32, p, u64, p]
    lib.rsd_kv4_append.argtypes = [p, p, i64, i64, p, i64, i64, i32, p, p, p, i32, p, p]
    lib.rsd_kv4_read.argtypes = [p, p, p, i32, p, p, i32, p]
    lib.rsd_kv4_attention.argtypes = [p, p, p, p, u64, p]
    lib.rsd_kv4_evict.argtypes = [p, p, i32, i32, p, u64, p]
    lib.rsd_w4_linear_workspace.argtypes = [i32, i32, i32, i32]
    lib.rsd_kv4_attention_workspace.argtypes = [p, p, i32]
    lib.rsd_kv4_evict_workspace.argtypes = [p, i32]
    f64, f32 = C.c_double, C.c_float
    lib.rsd_rope_frequencies.argtypes = [f64, i32, i32, f64, f64, f64, f64, p]
    lib.rsd_qk_rope.argtypes = [p, p, p, p, f32, i32, i32, i32, p]
    lib.rsd_kv_append.argtypes = [p, p, p, i64, i64, p, p, p, p, p, f32, i32, i32, p]
    lib.rsd_kv_read.argtypes = [p, p, p, i32, p, p, p]
    lib.rsd_kv_attention_workspace.argtypes = [p, p]
    lib.rsd_kv_attention.argtypes = [p, p, p, u64, p]
    for f in (lib.rsd_w4_linear_workspace, lib.rsd_kv4_attention_workspace, lib.rsd_kv4_evict_workspace, lib.rsd_kv_attention_workspace):
        f.restype = u64
    _lib = lib
    return lib


def _bad(text: str):
    raise _b.RsdError(_b.RSD_EINVAL, text)


def _done(rc: int, lib):
    if rc != 0:
        raise _b.RsdError(rc, lib.rsd_op_last_error().decode())


# the current device as a number, without the checks that a tensor on some GPU has passed already (0.1 instead of 0.4 us)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
# torch.cuda.current_stream(d).cuda_stream without the stream object (0.1 instead of 1.9 us, of the 6 to 10 that a small call takes)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda d: torch.cuda.current_stream(d).cuda_stream)


def _stream(t: torch.Tensor) -> int:
    """The current stream of the device that `t` lies on, which has to be the current device."""
    d = t.get_device()
    if d < 0 or d != _current_device():
        _bad(f"tensors have to be on the current device: got {t.device}")
    return _raw_stream(d)


def _on(name: str, t: torch.Tensor, like: torch.Tensor, dtype) -> None:
    if t.dtype is not dtype or t.device != like.device:
        _bad(f"{name}: {t.dtype} on {t.device}, needed {dtype} on {like.device}")


def _flat(name: str, t: torch.Tensor, like: torch.Tensor, dtype, shape) -> int:
    """Address of a contiguous tensor of the given type and shape."""
    if t.dtype is not dtype or t.device != like.device:
        _on(name, t, like, dtype)
    if t.shape != shape or not t.is_contiguous():
        _bad(f"{name}: shape {tuple(t.shape)}, needed {tuple(shape)}, contiguous")
    return t.data_ptr()


def _int(name: str, v, least: int) -> int:
    """A whole number from ``least`` on that the entry points' 32 bits hold (ctypes would take it modulo 2^32)."""
    try:
        n = index(v)
    except TypeError:
        n = -1
    if not least <= n < 1 << 31:
        _bad(f"{name}: {v!r}, needed a whole number from {least} to 2^31 - 1")
    return n


def _workspace(nbytes: int, like: torch.Tensor) -> Tuple[Optional[torch.Tensor], Optional[int]]:
    if not nbytes:
        return None, None
    w = like.new_empty(nbytes, dtype=_u8) if like.dtype is not _u8 else like.new_empty(nbytes)
    return w, w.data_ptr()


# ---- products with 4-bit weights

@lru_cache(maxsize=4096)
def _w4_bytes(rows: int, n: int, k: int, dtype: int) -> int:
    return (_lib or _load()).rsd_w4_linear_workspace(rows, n, k, dtype)


def rsd_w4_pack(w: torch.Tensor) -> W4:
    """Weights ``[n, k]`` (fp32 or bf16, rows k elements apart or more) in 4 bits."""
    lib = _lib or _load()
    if w.dim() != 2 or w.dtype not in _TYPE or w.numel() == 0 or (w.shape[1] > 1 and w.stride(1) != 1):
        _bad(f"w4_pack: {w.dtype} {tuple(w.shape)}, needed fp32 or bf16 [n, k] with contiguous rows")
    st = _stream(w)
    n, k = w.shape
    codes = torch.empty(-(-n // 16), -(-k // 128), 4, 16, 16, dtype=_u8, device=w.device)
    scales = torch.empty(-(-n // 16), -(-k // 512), 4, 16, 4, dtype=_u8, device=w.device)
    _done(lib.rsd_w4_pack(w.data_ptr(), _TYPE[w.dtype], w.stride(0) if n > 1 else k, n, k, codes.data_ptr(), scales.data_ptr(), st), lib)
    return W4(codes, scales, n, k)


def rsd_w4_linear(x: torch.Tensor, w4, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``x [rows, k] @ W.T`` for ``w4 = (codes, scales, n, k)``; ``[rows, n]`` of x's type (into ``out`` if given)."""
    lib = _lib or _load()
    codes, scales, n, k = w4
    t = _TYPE.get(x.dtype)
    if t is None or x.dim() != 2 or x.shape[1] != k or (k > 1 and x.stride(1) != 1):
        _bad(f"w4_linear: x is {x.dtype} {tuple(x.shape)}, needed fp32 or bf16 [rows, {k}] with contiguous rows")
    st = _stream(x)
    rows = x.shape[0]
    cp = _flat("w4 codes", codes, x, _u8, (-(-n // 16), -(-k // 128), 4, 16, 16))
    sp = _flat("w4 scales", scales, x, _u8, (-(-n // 16), -(-k // 512), 4, 16, 4))
    if out is None:
        out = x.new_empty(rows, n)
    else:
        _on("out", out, x, x.dtype)
        if out.shape != (rows, n) or (n > 1 and out.stride(1) != 1) or (rows > 1 and out.stride(0) < n):
            _bad(f"w4_linear: out has shape {tuple(out.shape)}, strides {out.stride()}, needed [{rows}, {n}] with contiguous rows")
    if rows == 0:
        return out
    nbytes = _w4_bytes(rows, n, k, t)
    ws, wp = _workspace(nbytes, x)
    _done(lib.rsd_w4_linear(C.byref(_W4(cp, sp, n, k)), x.data_ptr(), x.stride(0) if rows > 1 else k, out.data_ptr(),
                            out.stride(0) if rows > 1 else n, rows, t, wp, nbytes, st), lib)
    return out


# ---- the cache

def rsd_kv4_cache(batch: int, max_pages: int, n_pages: int, n_kv_heads: int, head_dim: int, device="cuda") -> Kv4Cache:
    """An empty cache: no sequence has pages or entries yet."""
    return Kv4Cache(torch.zeros(n_pages, n_kv_heads, 17 * head_dim, dtype=_u8, device=device),
                    torch.full((batch, max_pages), -1, dtype=_i32, device=device), torch.zeros(batch, dtype=_i32, device=device))


@lru_cache(maxsize=4096)
def _evict_bytes(n_pages, kv_heads, hd, batch, max_pages, budget) -> int:
    c = _Cache(16, 16, 16, n_pages, kv_heads, hd, batch, max_pages)
    return (_lib or _load()).rsd_kv4_evict_workspace(C.byref(c), budget)


def _cache(c) -> Tuple[_Cache, torch.Tensor, int]:
    pool, table, kv_len = c
    st = _stream(pool)
    shape, dev = pool.shape, pool.device
    if pool.dtype is not _u8 or len(shape) != 3 or shape[2] % 17 or not pool.is_contiguous():
        _bad(f"cache: the pool is {pool.dtype} {tuple(shape)}, needed uint8 [pages, kv heads, 17 * head_dim], contiguous")
    n, h, b = shape
    if table.dtype is not _i32 or table.device != dev or table.dim() != 2 or not table.is_contiguous():
        _bad(f"cache: the table is {table.dtype} {tuple(table.shape)} on {table.device}, needed int32 [batch, pages] on {dev}, contiguous")
    batch, max_pages = table.shape
    if kv_len.dtype is not _i32 or kv_len.device != dev or kv_len.shape != (batch,) or not kv_len.is_contiguous():
        _bad(f"cache: kv_len is {kv_len.dtype} {tuple(kv_len.shape)} on {kv_len.device}, needed int32 [{batch}] on {dev}, contiguous")
    return _Cache(pool.data_ptr(), table.data_ptr(), kv_len.data_ptr(), n, h, b // 17, batch, max_pages), pool, st


def _rows3(name: str, t: torch.Tensor, like: torch.Tensor, heads: Optional[int], hd: int) -> Tuple[int, int, int]:
    """Address, row and head stride of a [rows, heads, head_dim] tensor with contiguous heads."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or shape[2] != hd or (heads is not None and shape[1] != heads) or stride[2] != 1 or t.device != like.device:
        _bad(f"{name}: shape {tuple(t.shape)} on {t.device}, strides {t.stride()}, needed [rows, {heads or 'heads'}, {hd}], contiguous heads")
    return t.data_ptr(), stride[0], stride[1]


def _entries(name: str, t: torch.Tensor, c: _Cache, pool, dtype) -> Tuple[int, int, int]:
    """Address and strides of a [batch, n_kv_heads, slots] tensor."""
    shape, stride = t.shape, t.stride()
    if (t.dtype is not dtype or t.device != pool.device or len(shape) != 3 or shape[0] != c.batch or shape[1] != c.n_kv_heads
            or shape[2] < c.max_pages * PAGE or stride[2] != 1):
        _bad(f"{name}: {t.dtype} {tuple(shape)} on {t.device}, strides {stride}; needed {dtype} [{c.batch}, {c.n_kv_heads}, {c.max_pages * PAGE} or more], "
             f"contiguous in the slots, on {pool.device}")
    return t.data_ptr(), stride[0], stride[1]


def _book(c: _Cache, pool, scores, entry_pos) -> _Book:
    sp, sb, sh = (None, 0, 0) if scores is None else _entries("scores", scores, c, pool, _f32)
    pp, pb, ph = (None, 0, 0) if entry_pos is None else _entries("entry_pos", entry_pos, c, pool, _i32)
    return _Book(sp, pp, sb, sh, pb, ph)


def rsd_kv4_append(cache, k: torch.Tensor, v: torch.Tensor, seq: torch.Tensor, slot: torch.Tensor, position: Optional[torch.Tensor] = None,
                   entry_pos: Optional[torch.Tensor] = None, scores: Optional[torch.Tensor] = None) -> None:
    """Writes keys and values ``[rows, n_kv_heads, head_dim]`` into slot ``slot[i]`` of sequence ``seq[i]``; the entries' scores
    become 0 and their positions ``position``.  ``kv_len`` is left to the caller."""
    lib = _lib or _load()
    c, pool, st = _cache(cache)
    t = _TYPE.get(k.dtype)
    if t is None or v.dtype != k.dtype or v.shape != k.shape:
        _bad(f"append: k is {k.dtype} {tuple(k.shape)}, v {v.dtype} {tuple(v.shape)}; needed fp32 or bf16, alike")
    kp, kr, kh = _rows3("k", k, pool, c.n_kv_heads, c.head_dim)
    vp, vr, vh = _rows3("v", v, pool, c.n_kv_heads, c.head_dim)
    rows = k.shape[0]
    sp, lp = _flat("seq", seq, pool, _i32, (rows,)), _flat("slot", slot, pool, _i32, (rows,))
    pp = None if position is None else _flat("position", position, pool, _i32, (rows,))
    if entry_pos is not None and position is None:
        _bad("append: entry_pos is kept but no position is given")
    book = _book(c, pool, scores, entry_pos)
    if rows:
        _done(lib.rsd_kv4_append(C.byref(c), kp, kr, kh, vp, vr, vh, t, sp, lp, pp, rows, C.byref(book), st), lib)


def rsd_kv4_read(cache, seq: torch.Tensor, slot: torch.Tensor, head_dim: Optional[int] = None, dtype=torch.bfloat16) -> Tuple[torch.Tensor, torch.Tensor]:
    """Keys and values ``[rows, n_kv_heads, head_dim]`` of the entries (seq[i], slot[i]), as the cache holds them."""
    lib = _lib or _load()
    c, pool, st = _cache(cache)
    if dtype not in _TYPE or (head_dim is not None and head_dim != c.head_dim):
        _bad(f"read: {dtype}, head dimension {head_dim}; needed fp32 or bf16 and {c.head_dim}")
    if seq.dim() != 1:
        _bad(f"seq: shape {tuple(seq.shape)}, needed [rows]")
    rows = seq.shape[0]
    sp, lp = _flat("seq", seq, pool, _i32, (rows,)), _flat("slot", slot, pool, _i32, (rows,))
    k, v = pool.new_empty(2, rows, c.n_kv_heads, c.head_dim, dtype=dtype).unbind()
    if rows:
        _done(lib.rsd_kv4_read(C.byref(c), sp, lp, rows, k.data_ptr(), v.data_ptr(), _TYPE[dtype], st), lib)
    return k, v


@lru_cache(maxsize=4096)
def _attn_bytes(n_pages, kv_heads, hd, batch, max_pages, rows, max_rows, heads, max_kv, dtype, ragged, lse, scored) -> int:
    # the sizes only; the addresses stand for "given"
    c = _Cache(16, 16, 16, n_pages, kv_heads, hd, batch, max_pages)
    a = _Attn(16, 16, 16 if lse else None, 0, 0, 0, 0, 16 if ragged else None, rows, max_rows, heads, max_kv, dtype, 0.0)
    return (_lib or _load()).rsd_kv4_attention_workspace(C.byref(c), C.byref(a), int(scored))


def rsd_kv4_attention(cache, q: torch.Tensor, scale: float, *, row_start: Optional[torch.Tensor] = None, max_rows: Optional[int] = None,
                      max_kv: Optional[int] = None, scores: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                      want_lse: bool = False):
    """Attention of the rows ``q [rows, n_heads, head_dim]`` over the cache, their own entries included.

    Without ``row_start`` row b is sequence b's newest token; with it (``[batch + 1]`` int32) sequence b has the rows
    ``row_start[b] .. row_start[b + 1] - 1``, and each sees one entry more than the row before it.  ``max_rows`` bounds the rows of a sequence (default: all
    of them could be one's): rows beyond it are not computed, and the first ``max_rows`` are taken for the sequence's newest; their places in the result, like those of rows
    that no sequence has, are not written.  ``max_kv`` bounds ``kv_len`` (default: what the table can hold).  The tighter both are, the better the work is dealt.  ``scores`` ``[batch, n_kv_heads, slots]``
    grows by the weight each entry received.  ``out`` may be ``q`` itself, without ``scores``.  Returns ``out``, or ``(out, lse)`` with ``want_lse``."""
    lib = _lib or _load()
    c, pool, st = _cache(cache)
    t = _TYPE.get(q.dtype)
    if t is None:
        _bad(f"attention: q is {q.dtype}, needed fp32 or bf16")
    qp, qr, qh = _rows3("q", q, pool, None, c.head_dim)
    rows, heads = q.shape[0], q.shape[1]
    if heads == 0 or heads % c.n_kv_heads:
        _bad(f"attention: {heads} heads over {c.n_kv_heads} kv heads")
    if row_start is None:
        max_rows = 1 if max_rows is None else max_rows
        if rows != c.batch or max_rows != 1:
            _bad(f"attention: {rows} rows for {c.batch} sequences, max_rows {max_rows}, without row_start")
        rp = None
    else:
        max_rows = rows if max_rows is None else max_rows
        rp = _flat("row_start", row_start, pool, _i32, (c.batch + 1,))
    if out is None:
        out = q.new_empty(rows, heads, c.head_dim)
    elif out.dtype != q.dtype or out.shape != q.shape:
        _bad(f"attention: out is {out.dtype} {tuple(out.shape)}, needed {q.dtype} {tuple(q.shape)}")
    op, orow, oh = _rows3("out", out, pool, heads, c.head_dim)
    lse = q.new_empty(rows, heads, dtype=_f32) if want_lse else None
    if rows:
        max_rows = _int("attention: max_rows", max_rows, 1)
        cap = c.max_pages * PAGE
        max_kv = cap if max_kv is None else min(max(int(max_kv), -1), cap)
        nbytes = _attn_bytes(c.n_pages, c.n_kv_heads, c.head_dim, c.batch, c.max_pages, rows, max_rows, heads, max_kv, t, rp is not None, want_lse,
                             scores is not None)
        ws, wp = _workspace(nbytes, pool)
        a = _Attn(qp, op, lse.data_ptr() if want_lse else None, qr, qh, orow, oh, rp, rows, max_rows, heads, max_kv, t, scale)
        book = None if scores is None else C.byref(_book(c, pool, scores, None))
        _done(lib.rsd_kv4_attention(C.byref(c), C.byref(a), book, wp, nbytes, st), lib)
    return (out, lse) if want_lse else out


def rsd_kv4_evict(cache, scores: torch.Tensor, entry_pos: torch.Tensor, budget: int, recent: int = 0) -> None:
    """Cuts every (sequence, kv head) back to ``budget`` entries: the ones whose position is within ``recent`` of the newest, then
    those of the highest score.  The cache's pages and ``kv_len``, the scores and the positions are updated in place."""
    lib = _lib or _load()
    c, pool, st = _cache(cache)
    book = _book(c, pool, scores, entry_pos)
    budget, recent = _int("evict: budget", budget, 1), _int("evict: recent", recent, 0)
    if recent > budget:
        _bad(f"evict: budget {budget}, recent {recent}")
    nbytes = _evict_bytes(c.n_pages, c.n_kv_heads, c.head_dim, c.batch, c.max_pages, budget)
    ws, wp = _workspace(nbytes, pool)
    _done(lib.rsd_kv4_evict(C.byref(c), C.byref(book), budget, recent, wp, nbytes, st), lib)


# ---- norms and rotation of queries and keys

ROPE_KINDS = ("plain", "linear", "base", "parts")


def rsd_rope(rot_dim: int, theta: float = 1e4, *, scaling: str = "plain", factor: float = 1.0, original: float = 0.0, low: float = 1.0, high: float = 32.0,
             magnitude: Optional[float] = None, interleaved: bool = False, device="cuda") -> Rope:
    """A rotation of the first ``rot_dim`` dimensions of a head, with frequencies ``theta ** (-2 i / rot_dim)``.

    ``scaling`` fits them for contexts ``factor`` times as long: "linear" divides all by ``factor``, "base" raises theta so that the last one is, "parts" divides those that turn less than ``low``
    times over the ``original`` context, leaves those that turn more than ``high`` times, and goes over from one to the other between.  ``magnitude`` multiplies the rotated dimensions (default 1;
    0.1 log(factor) + 1 for "parts" with a factor above 1)."""
    lib = _lib or _load()
    rot_dim = _int("rope: rot_dim", rot_dim, 2)
    if scaling not in ROPE_KINDS:
        _bad(f"rope: scaling {scaling!r}, needed one of {', '.join(ROPE_KINDS)}")
    if rot_dim > 256:
        _bad(f"rope: rot_dim {rot_dim}, at most 256")
    freq = (C.c_double * (rot_dim // 2))()
    _done(lib.rsd_rope_frequencies(theta, rot_dim, ROPE_KINDS.index(scaling), factor, original, low, high, freq), lib)
    if magnitude is None:
        magnitude = 0.1 * math.log(factor) + 1.0 if scaling == "parts" and factor > 1 else 1.0
    return Rope(torch.tensor(list(freq), dtype=torch.float64, device=device), interleaved, magnitude)


def _packer(kind):
    """What packs the fields of a ctypes.Structure, in their order, into its bytes; one more, 0, stands for 4 bytes of padding at its end."""
    codes = "".join({C.c_void_p: "Q", C.c_int64: "q", C.c_int32: "i", C.c_float: "f"}[t] for _, t in kind._fields_)
    return struct.Struct("=" + codes + "i" * ((C.sizeof(kind) - struct.calcsize("=" + codes)) // 4)).pack


# The structures of these calls as bytes, packed field by field: 0.6 us against 1.8 for a ctypes.Structure of sixteen fields, of the 8 to 13 that a small call takes.
_ROPE_BYTES, _HEADS_BYTES, _KV_CACHE_BYTES, _KV_ATTN_BYTES = _packer(_Rope), _packer(_Heads), _packer(_KvCache), _packer(_KvAttn)
_f64 = torch.float64


def _rope(rope, device: int, hd: int) -> bytes:
    freq, interleaved, magnitude = rope
    shape = freq.shape
    if freq.dtype is not _f64 or freq.get_device() != device or len(shape) != 1 or not freq.is_contiguous() or not 2 <= 2 * shape[0] <= hd:
        _bad(f"rope: the frequencies are {freq.dtype} {tuple(shape)} on {freq.device}, needed float64 [1 .. {hd // 2}] on cuda:{device}, contiguous")
    try:
        return _ROPE_BYTES(freq.data_ptr(), 2 * shape[0], 1 if interleaved else 0, magnitude, 0)
    except (struct.error, OverflowError):
        _bad(f"rope: magnitude {magnitude!r}")


def _ints(name: str, t: torch.Tensor, device: int, rows: int) -> int:
    """Address of a contiguous int32 [rows]."""
    if t.dtype is not _i32 or t.shape != (rows,) or t.get_device() != device or not t.is_contiguous():
        _bad(f"{name}: {t.dtype} {tuple(t.shape)} on {t.device}, needed {_i32} [{rows}] on cuda:{device}, contiguous")
    return t.data_ptr()


def _heads(name: str, x: torch.Tensor, rows: int, hd: int, dtype, device: int, weight: Optional[torch.Tensor], out: Optional[torch.Tensor], writes: bool):
    """The heads of x [rows, heads, hd], and where they go: (structure, out)."""
    shape, stride = x.shape, x.stride()
    if len(stride) != 3 or stride[2] != 1 or shape[0] != rows or shape[2] != hd or x.dtype is not dtype or x.get_device() != device:
        _bad(f"{name}: {x.dtype} {tuple(shape)} on {x.device}, strides {stride}, needed {dtype} [{rows}, heads, {hd}] on cuda:{device}, contiguous heads")
    wp = 0
    if weight is not None:
        if weight.dtype is not dtype or weight.shape != (hd,) or not weight.is_contiguous() or weight.get_device() != device:
            _bad(f"{name}_weight: {weight.dtype} {tuple(weight.shape)} on {weight.device}, needed {dtype} [{hd}] on cuda:{device}, contiguous")
        wp = weight.data_ptr()
    if not writes:
        return _HEADS_BYTES(x.data_ptr(), 0, wp, stride[0], stride[1], 0, 0, shape[1], 0), None
    if out is None:
        heads = shape[1]
        out = x.new_empty(rows, heads, hd)
        return _HEADS_BYTES(x.data_ptr(), out.data_ptr(), wp, stride[0], stride[1], heads * hd, hd, heads, 0), out
    to = out.stride()
    if out.shape != shape or to[2] != 1 or out.dtype is not dtype or out.get_device() != device:
        _bad(f"{name}_out: {out.dtype} {tuple(out.shape)} on {out.device}, strides {to}, needed {dtype} {tuple(shape)} on cuda:{device}, contiguous heads")
    return _HEADS_BYTES(x.data_ptr(), out.data_ptr(), wp, stride[0], stride[1], to[0], to[1], shape[1], 0), out


def rsd_qk_rope(q: torch.Tensor, k: Optional[torch.Tensor], position: Optional[torch.Tensor], rope=None, *, q_weight: Optional[torch.Tensor] = None,
                k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
    """Heads ``q [rows, heads, head_dim]`` and ``k [rows, kv heads, head_dim]`` (may be None) normed over the head dimension, where they have a weight ``[head_dim]``, and
    rotated by ``rope`` (may be None) at ``position`` (int32 ``[rows]``).  Returns ``(q_out, k_out)``; an out may be its input itself."""
    lib = _lib or _load()
    dtype, shape = q.dtype, q.shape
    t = _TYPE.get(dtype)
    if t is None or len(shape) != 3 or shape[2] not in (32, 64, 128, 256) or shape[1] == 0:
        _bad(f"qk_rope: q is {dtype} {tuple(shape)}, needed fp32 or bf16 [rows, heads, 32, 64, 128 or 256]")
    st = _stream(q)
    rows, _, hd = shape
    device = q.get_device()
    qs, q_out = _heads("q", q, rows, hd, dtype, device, q_weight, q_out, True)
    ks = pp = rs = None
    if k is not None:
        ks, k_out = _heads("k", k, rows, hd, dtype, device, k_weight, k_out, True)
    elif k_weight is not None or k_out is not None:
        _bad("qk_rope: k_weight or k_out without k")
    if rope is not None:
        rs = _rope(rope, device, hd)
        if position is None:
            _bad("qk_rope: a rotation without positions")
        pp = _ints("position", position, device, rows)
    if rows:
        rc = lib.rsd_qk_rope(qs, ks, pp, rs, eps, rows, hd, t, st)
        if rc:
            _done(rc, lib)
    return q_out, k_out


# ---- the cache in bf16 or fp32

def rsd_kv_cache(batch: int, max_pages: int, n_pages: int, n_kv_heads: int, head_dim: int, dtype=torch.bfloat16, device="cuda") -> KvCache:
    """An empty cache: no sequence has pages or entries yet."""
    return KvCache(torch.zeros(n_pages, n_kv_heads, 2, PAGE * head_dim, dtype=dtype, device=device),
                   torch.full((batch, max_pages), -1, dtype=_i32, device=device), torch.zeros(batch, dtype=_i32, device=device))


def _kv_cache(c):
    """A cache as bytes, with what its calls go by: (bytes, pool, device, stream, (n_pages, n_kv_heads, head_dim, batch, max_pages, dtype))."""
    pool, table, kv_len = c
    st = _stream(pool)
    device = pool.get_device()
    shape, entries, t = pool.shape, table.shape, _TYPE.get(pool.dtype)
    if t is None or len(shape) != 4 or shape[2] != 2 or shape[3] % PAGE or not pool.is_contiguous():
        _bad(f"cache: the pool is {pool.dtype} {tuple(shape)}, needed fp32 or bf16 [pages, kv heads, 2, {PAGE} * head_dim], contiguous")
    if table.dtype is not _i32 or table.get_device() != device or len(entries) != 2 or not table.is_contiguous():
        _bad(f"cache: the table is {table.dtype} {tuple(entries)} on {table.device}, needed int32 [batch, pages] on {pool.device}, contiguous")
    batch, max_pages = entries
    sizes = (shape[0], shape[1], shape[3] // PAGE, batch, max_pages, t)
    if kv_len.dtype is not _i32 or kv_len.get_device() != device or kv_len.shape != (batch,) or not kv_len.is_contiguous():
        _bad(f"cache: kv_len is {kv_len.dtype} {tuple(kv_len.shape)} on {kv_len.device}, needed int32 [{batch}] on {pool.device}, contiguous")
    try:
        return _KV_CACHE_BYTES(pool.data_ptr(), table.data_ptr(), kv_len.data_ptr(), *sizes), pool, device, st, sizes
    except struct.error:
        _bad(f"cache: pool {tuple(shape)}, table {tuple(entries)}")


def rsd_kv_append(cache, k: torch.Tensor, v: torch.Tensor, seq: torch.Tensor, slot: torch.Tensor, *, position: Optional[torch.Tensor] = None, rope=None,
                  k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, q: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None,
                  q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """Writes keys and values ``[rows, n_kv_heads, head_dim]`` into slot ``slot[i]`` of sequence ``seq[i]``, the keys normed (with ``k_weight``) and rotated (with ``rope``, at
    ``position``) on their way; queries ``q [rows, heads, head_dim]`` of the same tokens go through the same in the same launch and are returned.  ``kv_len`` is left to the caller."""
    lib = _lib or _load()
    c, pool, device, st, (_, kv_heads, hd, _, _, _) = _kv_cache(cache)
    dtype, shape = k.dtype, k.shape
    t = _TYPE.get(dtype)
    if t is None or len(shape) != 3 or shape[1] != kv_heads:
        _bad(f"append: k is {dtype} {tuple(shape)}, needed fp32 or bf16 [rows, {kv_heads}, {hd}]")
    rows = shape[0]
    ks, _ = _heads("k", k, rows, hd, dtype, device, k_weight, None, False)
    stride = v.stride()
    if v.shape != shape or stride[2] != 1 or v.dtype is not dtype or v.get_device() != device:
        _bad(f"v: {v.dtype} {tuple(v.shape)} on {v.device}, strides {stride}, needed {dtype} {tuple(shape)} on cuda:{device}, contiguous heads")
    sp, lp = _ints("seq", seq, device, rows), _ints("slot", slot, device, rows)
    qs = pp = rs = None
    if q is not None:
        qs, q_out = _heads("q", q, rows, hd, dtype, device, q_weight, q_out, True)
    elif q_weight is not None or q_out is not None:
        _bad("append: q_weight or q_out without q")
    if rope is not None:
        rs = _rope(rope, device, hd)
        if position is None:
            _bad("append: a rotation without positions")
        pp = _ints("position", position, device, rows)
    if rows:
        rc = lib.rsd_kv_append(c, ks, v.data_ptr(), stride[0], stride[1], qs, sp, lp, pp, rs, eps, rows, t, st)
        if rc:
            _done(rc, lib)
    return q_out


def rsd_kv_read(cache, seq: torch.Tensor, slot: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """Keys and values ``[rows, n_kv_heads, head_dim]`` of the entries (seq[i], slot[i]); zeros where there is none."""
    lib = _lib or _load()
    c, pool, device, st, (_, kv_heads, hd, _, _, _) = _kv_cache(cache)
    if seq.dim() != 1:
        _bad(f"seq: shape {tuple(seq.shape)}, needed [rows]")
    rows = seq.shape[0]
    sp, lp = _ints("seq", seq, device, rows), _ints("slot", slot, device, rows)
    k, v = pool.new_empty(2, rows, kv_heads, hd).unbind()
    if rows:
        _done(lib.rsd_kv_read(c, sp, lp, rows, k.data_ptr(), v.data_ptr(), st), lib)
    return k, v


@lru_cache(maxsize=4096)
def _kv_attn_bytes(cache, rows, max_rows, heads, max_kv, window, sinks, dtype, ragged) -> int:
    # the sizes only; the addresses stand for "given"
    a = _KV_ATTN_BYTES(16, 16, 0, 0, 0, 0, 0, 16 if ragged else 0, rows, max_rows, heads, max_kv, window, sinks, dtype, 0.0)
    return (_lib or _load()).rsd_kv_attention_workspace(_KV_CACHE_BYTES(16, 16, 16, *cache), a)


def rsd_kv_attention(cache, q: torch.Tensor, scale: float, *, row_start: Optional[torch.Tensor] = None, max_rows: Optional[int] = None, max_kv: Optional[int] = None,
                     window: int = 0, sinks: int = 0, out: Optional[torch.Tensor] = None, want_lse: bool = False):
    """Attention of the rows ``q [rows, n_heads, head_dim]`` over the cache, their own entries included.

    Without ``row_start`` row b is sequence b's newest token; with it (``[batch + 1]`` int32) sequence b has the rows ``row_start[b] .. row_start[b + 1] - 1``, the last of which
    stands at its last entry.  ``max_rows`` bounds the rows of a sequence (default: all of them could be one's): rows beyond it are not computed, and the first ``max_rows`` are taken for the
    sequence's newest; their places in the result, like those of rows that no sequence has, are not written.  ``max_kv`` bounds ``kv_len`` (default: what the table can hold).  The tighter both are, the better the work is
    dealt (64 x 128 rows of 300 entries take 86 us, and 571 where ``max_rows`` is left out).  With ``window`` a row sees its own entry, the window - 1 before it, and a sequence's first ``sinks``.  ``out`` may be ``q`` itself.  Returns ``out``, or ``(out, lse)`` with ``want_lse``."""
    lib = _lib or _load()
    c, pool, device, st, sizes = _kv_cache(cache)
    _, kv_heads, hd, batch, max_pages, _ = sizes
    dtype, shape, stride = q.dtype, q.shape, q.stride()
    t = _TYPE.get(dtype)
    if t is None or len(shape) != 3 or stride[2] != 1 or shape[2] != hd or q.get_device() != device:
        _bad(f"attention: q is {dtype} {tuple(shape)} on {q.device}, strides {stride}, needed fp32 or bf16 [rows, heads, {hd}] on {pool.device}, contiguous heads")
    rows, heads, _ = shape
    if heads == 0 or kv_heads == 0 or heads % kv_heads:
        _bad(f"attention: {heads} heads over {kv_heads} kv heads")
    rp = 0
    if row_start is None:
        max_rows = 1 if max_rows is None else max_rows
        if rows != batch or max_rows != 1:
            _bad(f"attention: {rows} rows for {batch} sequences, max_rows {max_rows}, without row_start")
    else:
        max_rows = rows if max_rows is None else max_rows
        rp = _ints("row_start", row_start, device, batch + 1)
    if window.__class__ is not int or sinks.__class__ is not int or not 0 <= window < 1 << 31 or not 0 <= sinks < 1 << 31:
        window, sinks = _int("attention: window", window, 0), _int("attention: sinks", sinks, 0)
    if out is None:
        out = q.new_empty(rows, heads, hd)
        orow, oh = heads * hd, hd
    else:
        to = out.stride()
        if out.shape != shape or to[2] != 1 or out.dtype is not dtype or out.get_device() != device:
            _bad(f"attention: out is {out.dtype} {tuple(out.shape)} on {out.device}, strides {to}, needed {dtype} {tuple(shape)} on {pool.device}, contiguous heads")
        orow, oh, _ = to
    lse = q.new_empty((rows, heads), dtype=_f32) if want_lse else None
    if rows:
        if max_rows.__class__ is not int or not 1 <= max_rows < 1 << 31:
            max_rows = _int("attention: max_rows", max_rows, 1)
        cap = max_pages * PAGE
        max_kv = cap if max_kv is None else min(max(int(max_kv), -1), cap)
        try:
            a = _KV_ATTN_BYTES(q.data_ptr(), out.data_ptr(), lse.data_ptr() if want_lse else 0, stride[0], stride[1], orow, oh, rp, rows, max_rows, heads, max_kv, window, sinks, t, scale)
        except (struct.error, OverflowError):
            _bad(f"attention: {rows} rows of {heads} heads, scale {scale!r}")
        nbytes = _kv_attn_bytes(sizes, rows, max_rows, heads, max_kv, window, sinks, t, rp != 0)
        ws = pool.new_empty(nbytes, dtype=_u8) if nbytes else None
        rc = lib.rsd_kv_attention(c, a, ws.data_ptr() if nbytes else None, nbytes, st)
        if rc:
            _done(rc, lib)
    return (out, lse) if want_lse else out
