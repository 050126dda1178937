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

from . import _lib
from .attention import _call, _check_offsets, _check_tensor, _scale
from .build import CACHE_LIB

PAGE = 64

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


def _pool(cache, need_weight=False):
    """(struct ts_cache, device) of a SessionCache, whose tensors have to fit each other."""
    k, v, k_exp, v_exp, weight = cache
    for name, t, dtype in (("k", k, torch.float8_e4m3fn), ("v", v, torch.float8_e4m3fn), ("k_exp", k_exp, torch.uint8),
                           ("v_exp", v_exp, torch.uint8)):
        if not isinstance(t, torch.Tensor) or t.dtype != dtype or not t.is_cuda or not t.is_contiguous():
            raise ValueError("cache.%s must be a contiguous %s GPU tensor" % (name, dtype))
    shape = k.shape
    if len(shape) != 4 or shape[2] != PAGE or v.shape != shape or k_exp.shape != shape[:2] or v_exp.shape != shape[:2]:
        raise ValueError("a cache is k, v [pages, H, %d, d] and k_exp, v_exp [pages, H]" % PAGE)
    dev = k.device
    if v.device != dev or k_exp.device != dev or v_exp.device != dev:
        raise ValueError("a cache's tensors must be on one device")
    if weight is not None:
        _check_weight("cache.weight", weight, shape, dev)
    elif need_weight:
        raise ValueError("this call needs the cache's weight")
    pages, H, _, d = shape
    _lib.i32s(pages=pages, H=H, d=d)
    return _Pool(k.data_ptr(), v.data_ptr(), k_exp.data_ptr(), v_exp.data_ptr(),
                 None if weight is None else weight.data_ptr(), pages, H, d), dev


def _check_weight(name, t, shape, dev):
    if (not isinstance(t, torch.Tensor) or t.dtype != torch.float32 or t.shape != shape[:3] or t.device != dev
            or not t.is_contiguous()):
        raise ValueError("%s must be a contiguous float32 [pages, H, %d] tensor on the cache's device" % (name, PAGE))


def _check_ints(name, t, dim, dev):
    if not isinstance(t, torch.Tensor) or t.dtype != torch.int32 or t.dim() != dim or t.device != dev or not t.is_contiguous():
        raise ValueError("%s must be a contiguous int32 tensor with %d dims on the cache's device" % (name, dim))


def _sessions(table, lens, dev):
    """(nseq, width)"""
    _check_ints("table", table, 2, dev)
    _check_ints("lens", lens, 1, dev)
    if table.shape[0] != lens.shape[0]:
        raise ValueError("table and lens must have one row per session")
    return table.shape


def _rows(name, t, H, d, dev, groups=False):
    _check_tensor(name, t, 3)
    if t.device != dev or t.shape[2] != d or (t.shape[1] % H if groups else t.shape[1] != H) or t.shape[1] == 0:
        raise ValueError("%s must be [rows, %s, %d] on the cache's device" % (name, "a multiple of %d" % H if groups else H, d))


def _cu(cu, nseq, dev):
    _check_offsets("cu_seqlens", cu, dev)
    if cu.numel() != nseq + 1:
        raise ValueError("cu_seqlens must have one more entry than there are sessions")


def ts_cache_append(cache, k, v, cu_seqlens, max_seqlen, table, lens, out=None):
    """Appends each session's new tokens to its pages: k, v are bfloat16 [T, H, d], session s's rows
    [cu_seqlens[s], cu_seqlens[s+1]), at most max_seqlen of them, becoming its tokens lens[s], lens[s] + 1, ...
    of the pages table[s] (int32 [nseq, width]).  Returns the new lengths (int32 [nseq], or `out`)."""
    pool, dev = _pool(cache)
    nseq, width = _sessions(table, lens, dev)
    _rows("k", k, pool.H, pool.d, dev)
    _rows("v", v, pool.H, pool.d, dev)
    if v.shape != k.shape:
        raise ValueError("k and v must have one shape")
    _cu(cu_seqlens, nseq, dev)
    if out is None:
        out = torch.empty_like(lens)
    else:
        _check_ints("out", out, 1, dev)
        if out.shape != lens.shape:
            raise ValueError("out must match lens")
    _call(load_cache().ts_cache_append, dev, ctypes.addressof(pool), k.data_ptr(), v.data_ptr(), cu_seqlens.data_ptr(),
          table.data_ptr(), lens.data_ptr(), out.data_ptr(),
          *_lib.i32s(nseq=nseq, width=width, max_seqlen=max_seqlen, T=k.shape[0]))
    return out


def ts_cache_attn(q, cache, cu_seqlens, max_seqlen, table, lens, max_len, scale=None, out=None, lse=None,
                  return_lse=False, num_splits=0):
    """Attention of each session's query rows over its cached tokens: q is bfloat16 [T, Hq, d] with Hq a
    multiple of the cache's heads (query head hq reads cached head hq // (Hq // H)), session s's rows
    [cu_seqlens[s], cu_seqlens[s+1]), at most max_seqlen of them, over its lens[s] <= max_len tokens.  Returns o
    [T, Hq, d], or (o, lse) with lse float32 [T, Hq] when return_lse is set or an lse tensor is passed.
    num_splits: 0 lets the library choose, 1..64 forces that many page ranges per query tile."""
    pool, dev = _pool(cache)
    nseq, width = _sessions(table, lens, dev)
    _rows("q", q, pool.H, pool.d, dev, groups=True)
    _cu(cu_seqlens, nseq, dev)
    T, Hq, d = q.shape
    if out is None:
        out = torch.empty_like(q)
    else:
        _check_tensor("out", out, 3)
        if out.shape != q.shape or out.device != dev:
            raise ValueError("out must match q")
    if lse is None and return_lse:
        lse = torch.empty((T, Hq), dtype=torch.float32, device=dev)
    if lse is not None:
        _check_lse(lse, T, Hq, dev)
    sizes = _lib.i32s(nseq=nseq, width=width, max_seqlen=max_seqlen, max_len=max_len, T=T, Hq=Hq)
    num_splits = _lib.i32("num_splits", num_splits)
    lib = load_cache()
    with torch.cuda.device(dev):
        need = lib.ts_cache_attn_workspace(nseq, sizes[2], sizes[3], T, pool.H, Hq, d, num_splits)
    # from torch's allocator: the memory goes back to the current stream's pool (or, while a graph is
    # captured, the graph's own) when the call is enqueued, so no other work meets it
    work = torch.empty(need, dtype=torch.uint8, device=dev) if need > 0 else None
    _call(lib.ts_cache_attn, dev, ctypes.addressof(pool), q.data_ptr(), out.data_ptr(),
          None if lse is None else lse.data_ptr(), cu_seqlens.data_ptr(), table.data_ptr(), lens.data_ptr(),
          *sizes, _scale(scale, d), num_splits, None if work is None else work.data_ptr(), max(need, 0))
    return (out, lse) if lse is not None else out


def _check_lse(lse, T, Hq, dev):
    if (not isinstance(lse, torch.Tensor) or lse.dtype != torch.float32 or lse.shape != (T, Hq) or lse.device != dev
            or not lse.is_contiguous()):
        raise ValueError("lse must be a contiguous float32 [T, Hq] tensor on the cache's device")


def ts_cache_weigh(q, lse, cache, cu_seqlens, max_seqlen, table, lens, max_len, scale=None, out=None):
    """Adds to every cached token the attention weight that the queries give it: cache.weight plus, for
    each query row and head, exp(scale <q, k> - lse), with lse as ts_cache_attn returned it for these queries.
    In place, or into `out` (float32 [pages, H, 64], of which only the sessions' tokens are written); returns
    what it wrote to."""
    pool, dev = _pool(cache, need_weight=True)
    nseq, width = _sessions(table, lens, dev)
    _rows("q", q, pool.H, pool.d, dev, groups=True)
    _cu(cu_seqlens, nseq, dev)
    T, Hq, d = q.shape
    _check_lse(lse, T, Hq, dev)
    if out is None:
        out = cache[4]
    else:
        _check_weight("out", out, cache[0].shape, dev)
    _call(load_cache().ts_cache_weigh, dev, ctypes.addressof(pool), q.data_ptr(), lse.data_ptr(), cu_seqlens.data_ptr(),
          table.data_ptr(), lens.data_ptr(), out.data_ptr(),
          *_lib.i32s(nseq=nseq, width=width, max_seqlen=max_seqlen, max_len=max_len, T=T, Hq=Hq), _scale(scale, d))
    return out


def ts_cache_evict(cache, table, lens, max_len, new_table, keep, first=0, last=0, out=None, kept=None):
    """Cuts every session down to `keep` tokens per head, in the new pages new_table (int32 [nseq, width'],
    64 * width' >= keep): the first `first`, the last `last`, and of the others those with the largest
    weight (the earlier one of equals), in order.  Sessions of up to `keep` tokens keep them all.  Returns
    (new lengths int32 [nseq], kept positions int32 [nseq, H, keep], -1 past a session's new length)."""
    pool, dev = _pool(cache, need_weight=True)
    nseq, width = _sessions(table, lens, dev)
    _check_ints("new_table", new_table, 2, dev)
    keep = _lib.i32("keep", keep)
    if new_table.shape[0] != nseq:
        raise ValueError("new_table must have one row per session")
    if out is None:
        out = torch.empty_like(lens)
    else:
        _check_ints("out", out, 1, dev)
        if out.shape != lens.shape:
            raise ValueError("out must match lens")
    if kept is None:
        kept = torch.empty((nseq, pool.H, max(keep, 0)), dtype=torch.int32, device=dev)
    else:
        _check_ints("kept", kept, 3, dev)
        if kept.shape != (nseq, pool.H, keep):
            raise ValueError("kept must be [nseq, H, keep]")
    _call(load_cache().ts_cache_evict, dev, ctypes.addressof(pool), table.data_ptr(), lens.data_ptr(), new_table.data_ptr(),
          out.data_ptr(), kept.data_ptr(),
          *_lib.i32s(nseq=nseq, width=width, new_width=new_table.shape[1], max_len=max_len, keep=keep, first=first, last=last))
    return out, kept
