"""Torch-facing binding of the 8-bit session cache (include/ts_cache.h, libts_cache.so): argument
marshalling only.

A session's keys and values lie in pages of 64 tokens of one pool (SessionCache), found through a row of
page numbers; a chunk step of a session with a budget is

    lens = ts_cache_append(cache, k, v, cu, max_rows, table, lens)
    o, lse = ts_cache_attn(q, cache, cu, max_rows, table, lens, max_len, return_lse=True)
    ts_cache_weigh(q, lse, cache, cu, max_rows, table, lens, max_len)
    lens, kept = ts_cache_evict(cache, table, lens, max_len, new_table, keep, first, last)

Tables and lengths are int32 GPU tensors that the library reads on the device only; every call runs on
torch's current stream of the pool's device and does not wait for it.
"""
import ctypes
import os
from typing import NamedTuple

import torch
from torch import Tensor

from .attention import _call, _scale
from .build import CACHE_LIB

PAGE = 64
_E4M3, _U8, _I32, _F32, _BF16 = torch.float8_e4m3fn, torch.uint8, torch.int32, torch.float32, torch.bfloat16

_cache_lib = None


class _Pool(ctypes.Structure):
    """struct ts_cache"""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_exp", ctypes.c_void_p), ("v_exp", ctypes.c_void_p),
                ("weight", ctypes.c_void_p), ("pages", ctypes.c_int32), ("H", ctypes.c_int32), ("d", ctypes.c_int32)]


class SessionCache(NamedTuple):
    """The pool of pages.  k, v: float8_e4m3fn [pages, H, 64, d]; k_exp, v_exp: uint8 [pages, H], an element
    standing for e4m3 * 2^(exp - 127); weight: float32 [pages, H, 64], the attention weight that each token has
    collected, or None for a pool whose sessions are never weighed or evicted."""
    k: torch.Tensor
    v: torch.Tensor
    k_exp: torch.Tensor
    v_exp: torch.Tensor
    weight: torch.Tensor = None


def session_cache(pages, heads, head_dim, device="cuda", weight=True):
    """A zeroed SessionCache of `pages` pages on `device`."""
    def zeros(dtype, *shape):
        return torch.zeros(shape, dtype=dtype, device=device)
    values = [zeros(torch.uint8, pages, heads, PAGE, head_dim).view(torch.float8_e4m3fn) for _ in range(2)]
    return SessionCache(*values, zeros(torch.uint8, pages, heads), zeros(torch.uint8, pages, heads),
                        zeros(torch.float32, pages, heads, PAGE) if weight else None)


def load_cache():
    """The loaded library; raises if it has not been built (there is no fallback path)."""
    global _cache_lib
    if _cache_lib is not None:
        return _cache_lib
    if not os.path.exists(CACHE_LIB):
        raise ImportError("libts_cache.so is not built (%s); run __graft_entry__.build()" % CACHE_LIB)
    lib = ctypes.CDLL(CACHE_LIB)
    p, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    lib.ts_cache_append.argtypes = [p] * 7 + [i32] * 4 + [p]
    lib.ts_cache_attn.argtypes = [p] * 7 + [i32] * 6 + [f32, i32, p, i64, p]
    lib.ts_cache_attn_workspace.argtypes = [i32] * 8
    lib.ts_cache_attn_workspace.restype = i64
    lib.ts_cache_weigh.argtypes = [p] * 7 + [i32] * 6 + [f32, p]
    lib.ts_cache_evict.argtypes = [p] * 6 + [i32] * 7 + [p]
    for f in (lib.ts_cache_append, lib.ts_cache_attn, lib.ts_cache_weigh, lib.ts_cache_evict, lib.ts_cache_abi_version):
        f.restype = ctypes.c_int
    lib.ts_cache_abi_version.argtypes = []
    _cache_lib = lib
    return lib


def _not(t, dtype, dim, index):
    """Whether t is anything but a contiguous `dim`-dimensional tensor of this type on GPU `index`."""
    return (not isinstance(t, Tensor) or t.dtype is not dtype or t.dim() != dim or t.get_device() != index
            or not t.is_contiguous())


def _pool(cache, need_weight=False):
    """(struct ts_cache, device, its index) of a SessionCache, whose tensors have to fit each other."""
    k, v, k_exp, v_exp, weight = cache
    if not isinstance(k, Tensor) or not k.is_cuda:
        raise ValueError("cache.k must be a contiguous float8_e4m3fn GPU tensor")
    dev = k.device
    index = dev.index
    shape, scales = k.shape, k_exp.shape if isinstance(k_exp, Tensor) else None
    if _not(k, _E4M3, 4, index) or _not(v, _E4M3, 4, index):
        raise ValueError("cache.k and v must be contiguous float8_e4m3fn tensors [pages, H, %d, d] on one GPU" % PAGE)
    if _not(k_exp, _U8, 2, index) or _not(v_exp, _U8, 2, index):
        raise ValueError("cache.k_exp and v_exp must be contiguous uint8 tensors [pages, H] on the cache's GPU")
    pages, H, rows, d = shape
    if rows != PAGE or v.shape != shape or scales != shape[:2] or v_exp.shape != scales:
        raise ValueError("a cache is k, v [pages, H, %d, d] and k_exp, v_exp [pages, H]" % PAGE)
    if weight is not None:
        _check_weight("cache.weight", weight, shape, index)
    elif need_weight:
        raise ValueError("this call needs the cache's weight")
    _i32s("pages, H, d", pages, H, d)
    return _Pool(k.data_ptr(), v.data_ptr(), k_exp.data_ptr(), v_exp.data_ptr(),
                 None if weight is None else weight.data_ptr(), pages, H, d), dev, index


def _i32s(names, *values):
    """The sizes as C int32 arguments (ctypes would silently wrap a larger one)."""
    values = [int(x) for x in values]
    if min(values) < -(1 << 31) or max(values) >= 1 << 31:
        raise ValueError("%s = %s do not fit the C ABI's int32" % (names, values))
    return values


def _check_weight(name, t, shape, index):
    if _not(t, _F32, 3, index) or t.shape != shape[:3]:
        raise ValueError("%s must be a contiguous float32 [pages, H, %d] tensor on the cache's device" % (name, PAGE))


def _check_ints(name, t, dim, index):
    if _not(t, _I32, dim, index):
        raise ValueError("%s must be a contiguous int32 tensor with %d dims on the cache's device" % (name, dim))


def _sessions(cu, table, lens, index):
    """(nseq, width); cu, the sessions' rows, is None for a call without rows."""
    _check_ints("table", table, 2, index)
    _check_ints("lens", lens, 1, index)
    nseq, width = table.shape
    if lens.numel() != nseq:
        raise ValueError("table and lens must have one row per session")
    if cu is not None:
        _check_ints("cu_seqlens", cu, 1, index)
        if cu.numel() != nseq + 1:
            raise ValueError("cu_seqlens must have one more entry than there are sessions")
    return nseq, width


def _rows(name, t, H, d, index, groups=False):
    if not isinstance(t, Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if _not(t, _BF16, 3, index):
        raise ValueError("%s must be a contiguous bfloat16 tensor with 3 dims on the cache's device" % name)
    _, heads, channels = t.shape
    if channels != d or (heads % H if groups else heads != H) or heads == 0:
        raise ValueError("%s must be [rows, %s, %d]" % (name, "a multiple of %d" % H if groups else H, d))


def _lens_out(out, lens, index):
    if out is None:
        return torch.empty_like(lens)
    _check_ints("out", out, 1, index)
    if out.shape != lens.shape:
        raise ValueError("out must match lens")
    return out


def _check_lse(lse, T, Hq, index):
    if _not(lse, _F32, 2, index) or lse.shape != (T, Hq):
        raise ValueError("lse must be a contiguous float32 [T, Hq] tensor on the cache's device")


def ts_cache_append(cache, k, v, cu_seqlens, max_seqlen, table, lens, out=None):
    """Appends each session's new tokens to its pages: k, v are bfloat16 [T, H, d], session s's rows
    [cu_seqlens[s], cu_seqlens[s+1]), at most max_seqlen of them, becoming its tokens lens[s], lens[s] + 1, ...
    of the pages table[s] (int32 [nseq, width]).  Returns the new lengths (int32 [nseq], or `out`)."""
    pool, dev, index = _pool(cache)
    nseq, width = _sessions(cu_seqlens, table, lens, index)
    H, d = pool.H, pool.d
    _rows("k", k, H, d, index)
    _rows("v", v, H, d, index)
    T = k.shape[0]
    if v.shape[0] != T:
        raise ValueError("k and v must have one shape")
    out = _lens_out(out, lens, index)
    _call(load_cache().ts_cache_append, dev, ctypes.addressof(pool), k.data_ptr(), v.data_ptr(), cu_seqlens.data_ptr(),
          table.data_ptr(), lens.data_ptr(), out.data_ptr(),
          *_i32s("nseq, width, max_seqlen, T", nseq, width, max_seqlen, T))
    return out


def ts_cache_attn(q, cache, cu_seqlens, max_seqlen, table, lens, max_len, scale=None, out=None, lse=None,
                  return_lse=False, num_splits=0):
    """Attention of each session's query rows over its cached tokens: q is bfloat16 [T, Hq, d] with Hq a
    multiple of the cache's heads (query head hq reads cached head hq // (Hq // H)), session s's rows
    [cu_seqlens[s], cu_seqlens[s+1]), at most max_seqlen of them, over its lens[s] <= max_len tokens.  Returns o
    [T, Hq, d], or (o, lse) with lse float32 [T, Hq] when return_lse is set or an lse tensor is passed.
    num_splits: 0 lets the library choose, 1..64 forces that many page ranges per query tile."""
    pool, dev, index = _pool(cache)
    nseq, width = _sessions(cu_seqlens, table, lens, index)
    _rows("q", q, pool.H, pool.d, index, groups=True)
    T, Hq, d = q.shape
    if out is None:
        out = torch.empty_like(q)
    else:
        if _not(out, _BF16, 3, index) or out.shape != q.shape:
            raise ValueError("out must match q")
    if lse is None and return_lse:
        lse = q.new_empty((T, Hq), dtype=_F32)
    elif lse is not None:
        _check_lse(lse, T, Hq, index)
    sizes = _i32s("nseq, width, max_seqlen, max_len, T, Hq, num_splits", nseq, width, max_seqlen, max_len, T, Hq, num_splits)
    num_splits = sizes.pop()
    lib = load_cache()
    asked = nseq, sizes[2], sizes[3], T, pool.H, Hq, d, num_splits
    if torch.cuda.current_device() == index:
        need = lib.ts_cache_attn_workspace(*asked)
    else:
        with torch.cuda.device(dev):
            need = lib.ts_cache_attn_workspace(*asked)
    # from torch's allocator: the memory goes back to the current stream's pool (or, while a graph is
    # captured, the graph's own) when the call is enqueued, so no other work meets it
    work = q.new_empty(need, dtype=_U8) if need > 0 else None
    _call(lib.ts_cache_attn, dev, ctypes.addressof(pool), q.data_ptr(), out.data_ptr(),
          None if lse is None else lse.data_ptr(), cu_seqlens.data_ptr(), table.data_ptr(), lens.data_ptr(),
          *sizes, _scale(scale, d), num_splits, None if work is None else work.data_ptr(), max(need, 0))
    return (out, lse) if lse is not None else out


def ts_cache_weigh(q, lse, cache, cu_seqlens, max_seqlen, table, lens, max_len, scale=None, out=None):
    """Adds to every cached token the attention weight that the queries give it: cache.weight plus, for
    each query row and head, exp(scale <q, k> - lse), with lse as ts_cache_attn returned it for these queries.
    In place, or into `out` (float32 [pages, H, 64], of which only the sessions' tokens are written); returns
    what it wrote to."""
    pool, dev, index = _pool(cache, need_weight=True)
    nseq, width = _sessions(cu_seqlens, table, lens, index)
    _rows("q", q, pool.H, pool.d, index, groups=True)
    T, Hq, d = q.shape
    _check_lse(lse, T, Hq, index)
    if out is None:
        out = cache[4]
    else:
        _check_weight("out", out, cache[0].shape, index)
    _call(load_cache().ts_cache_weigh, dev, ctypes.addressof(pool), q.data_ptr(), lse.data_ptr(), cu_seqlens.data_ptr(),
          table.data_ptr(), lens.data_ptr(), out.data_ptr(),
          *_i32s("nseq, width, max_seqlen, max_len, T, Hq", nseq, width, max_seqlen, max_len, T, Hq), _scale(scale, d))
    return out


def ts_cache_evict(cache, table, lens, max_len, new_table, keep, first=0, last=0, out=None, kept=None):
    """Cuts every session down to `keep` tokens per head, in the new pages new_table (int32 [nseq, width'],
    64 * width' >= keep): the first `first`, the last `last`, and of the others those with the largest
    weight (the earlier one of equals), in order.  Sessions of up to `keep` tokens keep them all.  Returns
    (new lengths int32 [nseq], kept positions int32 [nseq, H, keep], -1 past a session's new length)."""
    pool, dev, index = _pool(cache, need_weight=True)
    nseq, width = _sessions(None, table, lens, index)
    _check_ints("new_table", new_table, 2, index)
    rows, new_width = new_table.shape
    if rows != nseq:
        raise ValueError("new_table must have one row per session")
    sizes = _i32s("nseq, width, new_width, max_len, keep, first, last", nseq, width, new_width, max_len, keep, first, last)
    keep = sizes[4]
    out = _lens_out(out, lens, index)
    if kept is None:
        kept = lens.new_empty((nseq, pool.H, max(keep, 0)))
    else:
        _check_ints("kept", kept, 3, index)
        if kept.shape != (nseq, pool.H, keep):
            raise ValueError("kept must be [nseq, H, keep]")
    _call(load_cache().ts_cache_evict, dev, ctypes.addressof(pool), table.data_ptr(), lens.data_ptr(), new_table.data_ptr(),
          out.data_ptr(), kept.data_ptr(), *sizes)
    return out, kept
