"""Torch-facing binding of what a transformer block does around attention (include/ts_block.h, libts_block.so): argument
marshalling only.

Serving:   q, k = ts_qk_rope(q, k, pos, rope, q_weight, k_weight)         (and then ts_attn_fwd*, or ts_cache_append)
Training:  o, lse = ts_attn_fwd_kvcache(q, k, v, cu, cu, L, L, return_lse=True)
           dq, dk, dv = ts_attn_bwd(d_o, q, k, v, o, lse, cu, cu, L, L)
           dq, dk, dq_weight, dk_weight = ts_qk_rope_bwd(dq, dk, q_in, k_in, pos, rope, q_weight, k_weight)

Every call runs on torch's current stream of its tensors' device and does not wait for it.
"""
import ctypes
import os
from typing import NamedTuple

import torch
from torch import Tensor

from . import _lib
from .attention import _call, _check_offsets, _scale
from .build import BLOCK_LIB

_I32, _F32, _F64, _U8, _BF16 = torch.int32, torch.float32, torch.float64, torch.uint8, torch.bfloat16

_block_lib = None


class Rope(NamedTuple):
    """A rotation by positions on three axes.  freq: float64 [d / 2] on the GPU, the angle of each pair per unit of
    position (0: the pair stays as it is); axes: how many of the pairs, in order, go by the first, the second and the
    third axis; interleaved: pair i is channels (2i, 2i + 1), else (i, i + d / 2)."""
    freq: torch.Tensor
    axes: tuple
    interleaved: bool = True


def rope(axes, theta=10000.0, interleaved=True, device="cuda"):
    """A Rope whose pair i of an axis' n turns by theta^(-i / n) per unit of position."""
    freq = [float(theta) ** (-i / n) for n in axes for i in range(n)]
    return Rope(torch.tensor(freq, dtype=_F64, device=device), tuple(axes), interleaved)


def load_block():
    """The loaded library; raises if it has not been built (there is no fallback path)."""
    global _block_lib
    if _block_lib is not None:
        return _block_lib
    if not os.path.exists(BLOCK_LIB):
        raise ImportError("libts_block.so is not built (%s); run __graft_entry__.build()" % BLOCK_LIB)
    lib = ctypes.CDLL(BLOCK_LIB)
    p, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    lib.ts_qk_rope.argtypes = [p] * 7 + [i32, i32, f32, p]
    lib.ts_qk_rope_bwd.argtypes = [p] * 11 + [i32, i32, f32, p, i64, p]
    lib.ts_qk_rope_bwd_workspace.argtypes = [i32] * 4
    lib.ts_qk_rope_bwd_workspace.restype = i64
    lib.ts_attn_bwd.argtypes = [p] * 11 + [i32] * 7 + [f32, i32, p, i64, p]
    lib.ts_attn_bwd_workspace.argtypes = [i32] * 8
    lib.ts_attn_bwd_workspace.restype = i64
    lib.ts_block_abi_version.argtypes = []
    for f in (lib.ts_qk_rope, lib.ts_qk_rope_bwd, lib.ts_attn_bwd, lib.ts_block_abi_version):
        f.restype = ctypes.c_int
    _block_lib = lib
    return lib


# A ts_rows is three 64-bit words here (p, stride, heads and padding), a ts_rope four (pos, freq, and the axes and the order in
# pairs of 32 bits): a call's structs are one array of them, which costs it a microsecond where eight ctypes structures cost six.
_Words = {n: ctypes.c_int64 * n for n in (10, 16, 22)}
_NO_ROWS = (0, 0, 0)


_TOP = (1 << 31) - 1


def _refuse_rows(name, t, shape):
    if not isinstance(t, Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if shape is not None and t.shape != shape:
        raise ValueError("%s must be %s" % (name, list(shape)))
    raise ValueError("%s must be a bfloat16 [T, heads, d] tensor on q's GPU" % name)


def _rows(name, t, shape, index):
    """The words of a tensor [T, heads, d] whose tokens may be any distance apart."""
    if not isinstance(t, Tensor) or t.dtype is not _BF16 or t.shape != shape or t.get_device() != index:
        _refuse_rows(name, t, shape)
    T, heads, d = shape
    stride, head, channel = t.stride()
    if T < 2:  # (the stride of a single token says nothing)
        stride = max(heads * d, 1)
    if (channel != 1 and d > 1 or head != d and heads > 1 or stride < heads * d) and T:
        raise ValueError("%s must have the heads of a token side by side" % name)
    return t.data_ptr(), stride, heads


def _out_rows(name, out, like, shape, index):
    """An output tensor, new or as given, and its words.  (empty_like takes a third less time than new_empty, and of `like`,
    whose heads lie side by side, it makes a tensor without gaps between the tokens.)"""
    if out is None:
        _, heads, d = shape
        out = torch.empty_like(like)
        return out, (out.data_ptr(), heads * d, heads)
    return out, _rows(name, out, shape, index)


def _first(name, t):
    """Shape, device and its index of the tensor that the others have to match, which is of rows of heads."""
    if not isinstance(t, Tensor) or t.dtype is not _BF16 or t.dim() != 3 or not t.is_cuda:
        _refuse_rows(name, t, None)
    shape = t.shape
    if max(shape) > _TOP:
        raise ValueError("%s = %s does not fit the C ABI's int32" % (name, list(shape)))
    dev = t.device
    return shape, dev, dev.index


def _beside(name, t, shape):
    """The shape of q's companion: its T and d, any heads."""
    if not isinstance(t, Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    other = t.shape
    if len(other) != 3 or other[0] != shape[0] or other[2] != shape[2] or other[1] > _TOP:
        raise ValueError("%s must be [%d, heads, %d]" % (name, shape[0], shape[2]))
    return other


def _weight(name, w, d, index):
    if w is None:
        return None
    if not isinstance(w, Tensor) or w.dtype is not _F32 or w.shape != (d,) or w.get_device() != index or not w.is_contiguous():
        raise ValueError("%s must be a contiguous float32 [%d] tensor on q's device" % (name, d))
    return w.data_ptr()


def _rope_words(pos, r, T, d, index):
    if r is None:
        if pos is not None:
            raise ValueError("positions need a rope")
        return 0, 0, 0, 0
    freq, axes, interleaved = r
    if not isinstance(pos, Tensor) or pos.dtype is not _I32 or pos.shape != (T, 3) or pos.get_device() != index or not pos.is_contiguous():
        raise ValueError("pos must be a contiguous int32 [T, 3] tensor on q's device")
    if (not isinstance(freq, Tensor) or freq.dtype is not _F64 or freq.shape != (d // 2,) or freq.get_device() != index
            or not freq.is_contiguous()):
        raise ValueError("rope.freq must be a contiguous float64 [d / 2] tensor on q's device")
    a, b, c = axes
    if min(a, b, c) < 0 or a + b + c != d // 2:
        raise ValueError("rope.axes must be three numbers of pairs, %d in all" % (d // 2))
    return pos.data_ptr(), freq.data_ptr(), a | b << 32, c | (1 << 32 if interleaved else 0)


def ts_qk_rope(q, k, pos=None, rope=None, q_weight=None, k_weight=None, eps=1e-6, q_out=None, k_out=None):
    """Norm and rotation of queries and keys in one pass: q is bfloat16 [T, Hq, d], k [T, Hk, d] or None, the heads of a
    token side by side, tokens any distance apart (views of a fused projection).  Where there are weights (float32 [d]) each head is
    divided by its root mean square, sqrt(mean + eps), and multiplied by them; where there is a rope its pairs turn by pos
    (int32 [T, 3]: time, height, width).  Returns (q_out, k_out), new or as given; they may be q and k themselves."""
    shape, dev, index = _first("q", q)
    T, _, d = shape
    k_at = ko_at = None
    rows = _rows("q", q, shape, index)
    q_out, out = _out_rows("q_out", q_out, q, shape, index)
    head = *rows, *out, *_rope_words(pos, rope, T, d, index)
    if k is not None:
        k_shape = _beside("k", k, shape)
        rows = _rows("k", k, k_shape, index)
        k_out, out = _out_rows("k_out", k_out, k, k_shape, index)
        words = _Words[16](*head, *rows, *out)
        at = ctypes.addressof(words)
        k_at, ko_at = at + 80, at + 104
    else:
        if k_out is not None or k_weight is not None:
            raise ValueError("k_out and k_weight need k")
        words = _Words[10](*head)
        at = ctypes.addressof(words)
    _call(load_block().ts_qk_rope, dev, at, k_at, at + 24, ko_at, _weight("q_weight", q_weight, d, index),
          _weight("k_weight", k_weight, d, index), None if rope is None else at + 48, T, d, eps)
    return q_out, k_out


def ts_qk_rope_bwd(dq_out, dk_out, q, k, pos=None, rope=None, q_weight=None, k_weight=None, eps=1e-6, dq=None, dk=None,
                   dq_weight=None, dk_weight=None):
    """The gradients of ts_qk_rope(q, k, pos, rope, q_weight, k_weight, eps) from those of its results: returns (dq, dk,
    dq_weight, dk_weight), the last two float32 [d], or None where the weight is (q or k may be None too there).  dk_out
    is None where k was.  dq and dk may be dq_out and dk_out, or q and k, themselves."""
    shape, dev, index = _first("dq_out", dq_out)
    T, Hq, d = shape
    Hk = 0
    go = _rows("dq_out", dq_out, shape, index)
    dq, gq = _out_rows("dq", dq, dq_out, shape, index)
    ho = hk = k_rows = q_rows = _NO_ROWS
    if dk_out is not None:
        k_shape = _beside("dk_out", dk_out, shape)
        Hk = k_shape[1]
        ho = _rows("dk_out", dk_out, k_shape, index)
        dk, hk = _out_rows("dk", dk, dk_out, k_shape, index)
    elif k is not None or dk is not None or k_weight is not None:
        raise ValueError("k, dk and k's weight need dk_out")
    if q_weight is not None:
        q_rows = _rows("q", q, shape, index)
        wq = _weight("q_weight", q_weight, d, index)
        if dq_weight is None:
            dq_weight = torch.empty_like(q_weight)
        gwq = _weight("dq_weight", dq_weight, d, index)
    else:
        if dq_weight is not None:
            raise ValueError("dq_weight needs q_weight")
        wq = gwq = None
    if k_weight is not None:
        k_rows = _rows("k", k, k_shape, index)
        wk = _weight("k_weight", k_weight, d, index)
        if dk_weight is None:
            dk_weight = torch.empty_like(k_weight)
        gwk = _weight("dk_weight", dk_weight, d, index)
    else:
        if dk_weight is not None:
            raise ValueError("dk_weight needs k_weight")
        wk = gwk = None
    words = _Words[22](*go, *gq, *_rope_words(pos, rope, T, d, index), *ho, *hk, *q_rows, *k_rows)
    at = ctypes.addressof(words)
    lib = load_block()
    need = lib.ts_qk_rope_bwd_workspace(T, Hq, Hk, d) if wq or wk else 0
    # from torch's allocator: the memory goes back to the current stream's pool (or, while a graph is
    # captured, the graph's own) when the call is enqueued, so no other work meets it
    work = dq_out.new_empty(need, dtype=_U8) if need > 0 else None
    _call(lib.ts_qk_rope_bwd, dev, at, at + 80 if Hk else None, at + 128 if wq else None, at + 152 if wk else None, at + 24,
          at + 104 if Hk else None, wq, wk, gwq, gwk, None if rope is None else at + 48, T, d, eps,
          None if work is None else work.data_ptr(), need)
    return dq, dk, dq_weight, dk_weight


def _like(name, t, shape, index, what):
    if not isinstance(t, Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.dtype is not _BF16 or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        raise ValueError("%s must be a contiguous bfloat16 tensor of %s" % (name, what))
    return t


def ts_attn_bwd(d_o, q, k, v, o, lse, cu_seqlens_q, cu_seqlens_k, max_seqlen_q, max_seqlen_k, scale=None, dq=None, dk=None,
                dv=None, num_splits=0):
    """The gradients (dq, dk, dv) of o, lse = ts_attn_fwd_kvcache(q, k, v, cu_seqlens_q, cu_seqlens_k, max_seqlen_q,
    max_seqlen_k, scale, return_lse=True), and so of the packed and the dense call, from d_o, the gradient of o: all bfloat16,
    d_o, o and dq as q [Tq, H, d], dk and dv as k [Tk, H, d], contiguous.  The offsets cover all rows.
    num_splits: 0 lets the library divide the work, 1..16 forces that many ranges of the other side's rows per tile."""
    shape_q, dev, index = _first("q", q)
    Tq, H, d = shape_q
    for name, t in (("q", q), ("o", o), ("d_o", d_o)):
        _like(name, t, shape_q, index, "q's shape and device")
    shape_k = _beside("k", k, (k.shape[0] if isinstance(k, Tensor) and k.dim() == 3 else 0, H, d))
    if shape_k[1] != H:
        raise ValueError("k and v must be [Tk, H, d] with q's H and d")
    for name, t in (("k", k), ("v", v)):
        _like(name, t, shape_k, index, "[Tk, H, d] with q's H, d and device")
    _check_offsets("cu_seqlens_q", cu_seqlens_q, dev)
    _check_offsets("cu_seqlens_k", cu_seqlens_k, dev)
    nseq = cu_seqlens_q.numel() - 1
    if cu_seqlens_k.numel() != nseq + 1:
        raise ValueError("cu_seqlens_q and cu_seqlens_k must have the same length")
    if nseq == 0 and (Tq or shape_k[0]):
        raise ValueError("the offsets have no segment, and q or k have rows")
    if (not isinstance(lse, Tensor) or lse.dtype is not _F32 or lse.shape != (Tq, H) or lse.get_device() != index
            or not lse.is_contiguous()):
        raise ValueError("lse must be a contiguous float32 [Tq, H] tensor on q's device")
    dq = torch.empty_like(q) if dq is None else _like("dq", dq, shape_q, index, "q's shape and device")
    dk = torch.empty_like(k) if dk is None else _like("dk", dk, shape_k, index, "k's shape and device")
    dv = torch.empty_like(v) if dv is None else _like("dv", dv, shape_k, index, "v's shape and device")
    *sizes, num_splits = _lib.i32s(nseq=nseq, max_seqlen_q=max_seqlen_q, max_seqlen_k=max_seqlen_k, Tq=Tq, Tk=shape_k[0], H=H, d=d,
                                   num_splits=num_splits)
    lib = load_block()
    if torch.cuda.current_device() == index:
        need = lib.ts_attn_bwd_workspace(*sizes, num_splits)
    else:
        with torch.cuda.device(dev):
            need = lib.ts_attn_bwd_workspace(*sizes, num_splits)
    work = q.new_empty(need, dtype=_U8) if need > 0 else None  # (as in ts_qk_rope_bwd)
    _call(lib.ts_attn_bwd, dev, d_o.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
          dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), cu_seqlens_q.data_ptr(), cu_seqlens_k.data_ptr(), *sizes,
          _scale(scale, d), num_splits, None if work is None else work.data_ptr(), need)
    return dq, dk, dv
