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
from .attention import _call, _check_offsets, _check_tensor, _scale
from .build import BLOCK_LIB

_I32, _F32, _F64, _U8, _BF16 = torch.int32, torch.float32, torch.float64, torch.uint8, torch.bfloat16

_block_lib = None


class _Rows(ctypes.Structure):
    """struct ts_rows"""
    _fields_ = [("p", ctypes.c_void_p), ("stride", ctypes.c_int64), ("heads", ctypes.c_int32)]


class _Rope(ctypes.Structure):
    """struct ts_rope"""
    _fields_ = [("pos", ctypes.c_void_p), ("freq", ctypes.c_void_p), ("axes", ctypes.c_int32 * 3), ("interleaved", ctypes.c_int32)]


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


def _rows(name, t, device, shape=None):
    """(struct ts_rows, its address) of a tensor [T, heads, d] whose tokens may be any distance apart."""
    if not isinstance(t, Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.dtype is not _BF16 or t.dim() != 3 or not t.is_cuda or (device is not None and t.device != device):
        raise ValueError("%s must be a bfloat16 [T, heads, d] tensor on q's GPU" % name)
    if shape is not None and t.shape != shape:
        raise ValueError("%s must be %s" % (name, list(shape)))
    T, heads, d = t.shape
    stride, head, channel = t.stride()
    if T < 2:  # (the stride of a single token says nothing)
        stride = max(heads * d, 1)
    if T and ((heads > 1 and head != d) or (d > 1 and channel != 1) or stride < heads * d):
        raise ValueError("%s must have the heads of a token side by side" % name)
    r = _Rows(t.data_ptr(), stride, heads)
    return r, ctypes.addressof(r)


def _out(name, out, like):
    return torch.empty(like.shape, dtype=_BF16, device=like.device) if out is None else out


def _weight(name, w, d, device):
    if w is None:
        return None
    if not isinstance(w, Tensor) or w.dtype is not _F32 or w.shape != (d,) or w.device != device or not w.is_contiguous():
        raise ValueError("%s must be a contiguous float32 [%d] tensor on q's device" % (name, d))
    return w.data_ptr()


def _rope_struct(pos, r, T, d, device):
    """(struct ts_rope, its address), or (None, None)."""
    if r is None:
        if pos is not None:
            raise ValueError("positions need a rope")
        return None, None
    freq, axes, interleaved = r
    if not isinstance(pos, Tensor) or pos.dtype is not _I32 or pos.shape != (T, 3) or pos.device != device or not pos.is_contiguous():
        raise ValueError("pos must be a contiguous int32 [T, 3] tensor on q's device")
    if not isinstance(freq, Tensor) or freq.dtype is not _F64 or freq.shape != (d // 2,) or freq.device != device or not freq.is_contiguous():
        raise ValueError("rope.freq must be a contiguous float64 [d / 2] tensor on q's device")
    if len(axes) != 3 or min(axes) < 0 or sum(axes) != d // 2:
        raise ValueError("rope.axes must be three numbers of pairs, %d in all" % (d // 2))
    s = _Rope(pos.data_ptr(), freq.data_ptr(), (ctypes.c_int32 * 3)(*axes), bool(interleaved))
    return s, ctypes.addressof(s)


def ts_qk_rope(q, k, pos=None, rope=None, q_weight=None, k_weight=None, eps=1e-6, q_out=None, k_out=None):
    """Norm and rotation of queries and keys in one pass: q is bfloat16 [T, Hq, d], k [T, Hk, d] or None, the heads of a
    token side by side, tokens any distance apart (views of a fused projection).  Where there are weights (float32 [d]) each head is
    divided by its root mean square, sqrt(mean + eps), and multiplied by them; where there is a rope its pairs turn by pos
    (int32 [T, 3]: time, height, width).  Returns (q_out, k_out), new or as given; they may be q and k themselves."""
    qs, q_at = _rows("q", q, None)
    T, _, d = q.shape
    dev = q.device
    ks = k_at = ko = ko_at = None
    if k is not None:
        ks, k_at = _rows("k", k, dev, (T, k.shape[1] if k.dim() == 3 else 0, d))
        k_out = _out("k_out", k_out, k)
        ko, ko_at = _rows("k_out", k_out, dev, k.shape)
    elif k_out is not None or k_weight is not None:
        raise ValueError("k_out and k_weight need k")
    q_out = _out("q_out", q_out, q)
    qo, qo_at = _rows("q_out", q_out, dev, q.shape)
    r, r_at = _rope_struct(pos, rope, T, d, dev)
    _call(load_block().ts_qk_rope, dev, q_at, k_at, qo_at, ko_at, _weight("q_weight", q_weight, d, dev),
          _weight("k_weight", k_weight, d, dev), r_at, *_lib.i32s(T=T, d=d), eps)
    return q_out, k_out


def ts_qk_rope_bwd(dq_out, dk_out, q, k, pos=None, rope=None, q_weight=None, k_weight=None, eps=1e-6, dq=None, dk=None,
                   dq_weight=None, dk_weight=None):
    """The gradients of ts_qk_rope(q, k, pos, rope, q_weight, k_weight, eps) from those of its results: returns (dq, dk,
    dq_weight, dk_weight), the last two float32 [d], or None where the weight is (q or k may be None too there).  dk_out
    is None where k was.  dq and dk may be dq_out and dk_out, or q and k, themselves."""
    go, go_at = _rows("dq_out", dq_out, None)
    T, Hq, d = dq_out.shape
    dev = dq_out.device
    Hk = 0
    ho = ho_at = gk = gk_at = q_at = k_at = None
    if dk_out is not None:
        ho, ho_at = _rows("dk_out", dk_out, dev, (T, dk_out.shape[1] if dk_out.dim() == 3 else 0, d))
        Hk = dk_out.shape[1]
        dk = _out("dk", dk, dk_out)
        gk, gk_at = _rows("dk", dk, dev, dk_out.shape)
    elif k is not None or dk is not None or k_weight is not None or dk_weight is not None:
        raise ValueError("k, dk and k's weight need dk_out")
    dq = _out("dq", dq, dq_out)
    gq, gq_at = _rows("dq", dq, dev, dq_out.shape)
    if q_weight is not None:
        qs, q_at = _rows("q", q, dev, dq_out.shape)
        dq_weight = torch.empty_like(q_weight) if dq_weight is None else dq_weight
    elif dq_weight is not None:
        raise ValueError("dq_weight needs q_weight")
    if k_weight is not None:
        ks, k_at = _rows("k", k, dev, dk_out.shape)
        dk_weight = torch.empty_like(k_weight) if dk_weight is None else dk_weight
    elif dk_weight is not None:
        raise ValueError("dk_weight needs k_weight")
    r, r_at = _rope_struct(pos, rope, T, d, dev)
    weights = [_weight(n, w, d, dev) for n, w in (("q_weight", q_weight), ("k_weight", k_weight), ("dq_weight", dq_weight),
                                                  ("dk_weight", dk_weight))]
    sizes = _lib.i32s(T=T, d=d)
    lib = load_block()
    need = lib.ts_qk_rope_bwd_workspace(T, Hq, Hk, d) if weights[0] or weights[1] else 0
    # from torch's allocator: the memory goes back to the current stream's pool (or, while a graph is
    # captured, the graph's own) when the call is enqueued, so no other work meets it
    work = dq_out.new_empty(need, dtype=_U8) if need > 0 else None
    _call(lib.ts_qk_rope_bwd, dev, go_at, ho_at, q_at, k_at, gq_at, gk_at, *weights, r_at, *sizes, eps,
          None if work is None else work.data_ptr(), need)
    return dq, dk, dq_weight, dk_weight


def ts_attn_bwd(d_o, q, k, v, o, lse, cu_seqlens_q, cu_seqlens_k, max_seqlen_q, max_seqlen_k, scale=None, dq=None, dk=None,
                dv=None, num_splits=0):
    """The gradients (dq, dk, dv) of o, lse = ts_attn_fwd_kvcache(q, k, v, cu_seqlens_q, cu_seqlens_k, max_seqlen_q,
    max_seqlen_k, scale, return_lse=True), and so of the packed and the dense call, from d_o, the gradient of o: all bfloat16,
    d_o, o and dq as q [Tq, H, d], dk and dv as k [Tk, H, d], contiguous.  Rows of no segment are not written.
    num_splits: 0 lets the library divide the work, 1..16 forces that many ranges of the other side's rows per tile."""
    for name, t in (("q", q), ("k", k), ("v", v), ("o", o), ("d_o", d_o)):
        _check_tensor(name, t, 3)
    dev, shape_q, shape_k = q.device, q.shape, k.shape
    if o.shape != shape_q or d_o.shape != shape_q or o.device != dev or d_o.device != dev:
        raise ValueError("o and d_o must match q")
    if v.shape != shape_k or shape_k[1:] != shape_q[1:] or k.device != dev or v.device != dev:
        raise ValueError("k and v must be [Tk, H, d] with q's H, d and device")
    _check_offsets("cu_seqlens_q", cu_seqlens_q, dev)
    _check_offsets("cu_seqlens_k", cu_seqlens_k, dev)
    nseq = cu_seqlens_q.numel() - 1
    if cu_seqlens_k.numel() != nseq + 1:
        raise ValueError("cu_seqlens_q and cu_seqlens_k must have the same length")
    Tq, H, d = shape_q
    if not isinstance(lse, Tensor) or lse.dtype is not _F32 or lse.shape != (Tq, H) or lse.device != dev or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous float32 [Tq, H] tensor on q's device")
    outs = []
    for name, t, like in (("dq", dq, q), ("dk", dk, k), ("dv", dv, v)):
        if t is None:
            t = torch.empty_like(like)
        else:
            _check_tensor(name, t, 3)
            if t.shape != like.shape or t.device != dev:
                raise ValueError("%s must match %s" % (name, name[1]))
        outs.append(t)
    *sizes, num_splits = _lib.i32s(nseq=nseq, max_seqlen_q=max_seqlen_q, max_seqlen_k=max_seqlen_k, Tq=Tq, Tk=shape_k[0], H=H, d=d,
                                   num_splits=num_splits)
    lib = load_block()
    if torch.cuda.current_device() == dev.index:
        need = lib.ts_attn_bwd_workspace(*sizes, num_splits)
    else:
        with torch.cuda.device(dev):
            need = lib.ts_attn_bwd_workspace(*sizes, num_splits)
    work = q.new_empty(need, dtype=_U8) if need > 0 else None  # (as in ts_qk_rope_bwd)
    _call(lib.ts_attn_bwd, dev, d_o.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
          outs[0].data_ptr(), outs[1].data_ptr(), outs[2].data_ptr(), cu_seqlens_q.data_ptr(), cu_seqlens_k.data_ptr(), *sizes,
          _scale(scale, d), num_splits, None if work is None else work.data_ptr(), need)
    return tuple(outs)
