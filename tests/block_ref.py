"""Plain 64-bit forms of the transformer block's calls (include/ts_block.h), one segment and one head at a time, and how far results
rounded to bfloat16 may be from them.  Used by tests/test_block_ref.py and tests/test_gpu_block.py; shares no code with
the library."""
import math

import numpy as np
import torch

HALF = 2.0 ** -8  # half a bfloat16 step, relative to the value
# of sums and functions in 32 bits, relative to the sum of their terms' magnitudes: 2^-24 a rounding, at most 256 of
# them in a chain (128 channels, each a product and a sum)
FINE = 2.0 ** -16
LEAST = 2.0 ** -126  # the least normal number of both types


def angles(pos, freq, axes):
    """[T, d / 2]"""
    axis = np.repeat(np.arange(3), axes)
    return pos.double()[:, torch.as_tensor(axis, device=pos.device)] * freq.double()


def split(x, interleaved):
    return (x[..., 0::2], x[..., 1::2]) if interleaved else x.chunk(2, -1)


def join(a, b, interleaved):
    return torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)


def rope(x, weight, angle, interleaved, eps):
    """x [T, H, d] in 64 bits (differentiable); angle [T, d / 2] or None."""
    if weight is not None:
        x = x * weight / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    if angle is None:
        return x
    a, b = split(x, interleaved)
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    return join(a * c - b * s, a * s + b * c, interleaved)


def rope_slack(x, weight, angle, interleaved, eps):
    """The sum of magnitudes whose 32-bit rounding an element of rope's result has."""
    if weight is not None:
        x = x * weight / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    if angle is None:
        return x.abs()
    a, b = split(x, interleaved)
    m = a.abs() + b.abs()
    return join(m, m, interleaved)


def rope_bwd(dy, x, weight, angle, interleaved, eps):
    """(dx, dweight or None), and the magnitudes that go into each."""
    d = dy.shape[-1]
    g, m = dy, dy.abs()
    if angle is not None:
        a, b = split(dy, interleaved)
        c, s = angle.cos()[:, None], angle.sin()[:, None]
        g = join(a * c + b * s, b * c - a * s, interleaved)
        m = join(a.abs() + b.abs(), a.abs() + b.abs(), interleaved)
    if weight is None:
        return g, None, m, None
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    n = x * r
    dot = (g * weight * n).sum(-1, keepdim=True) / d
    dx = r * (g * weight - n * dot)
    mags = r * (m * weight.abs() + n.abs() * (m * weight.abs() * n.abs()).sum(-1, keepdim=True) / d)
    return dx, (g * n).sum((0, 1)), mags, (m * n.abs()).sum((0, 1))


def attn(q, k, v, scale):
    """(o, lse) of one segment and head."""
    if k.shape[0] == 0:
        return torch.zeros_like(q), torch.full((q.shape[0],), -math.inf, dtype=q.dtype, device=q.device)
    x = scale * (q @ k.T)
    return torch.softmax(x, 1) @ v, torch.logsumexp(x, 1)


def attn_bwd(d_o, q, k, v, o, lse, scale):
    """(dq, dk, dv) of one segment and head and how far each element may be off.  What is below 2^-126 in 32 bits or bfloat16 may
    count as 0 (the GPU's exp2 and matrix products have no smaller numbers): P by 2^-126, S by that times what it is P times
    of, and by 2^-126.  P and S = P (d_o v - D) are rounded to
    bfloat16 (each off by HALF at most, one way or the other: of n such terms t the sum is off by HALF sum |t| at the very most, and
    by 6 sqrt(sum t^2) HALF in one of 10^7 cases), all before that are sums in 32 bits, the results are rounded
    once more."""
    if q.shape[0] == 0 or k.shape[0] == 0:
        z = [torch.zeros_like(x) for x in (q, k, v)]
        return z, [x.clone() for x in z]
    p = torch.exp(scale * (q @ k.T) - lse[:, None])
    t = d_o @ v.T - (d_o * o).sum(1, keepdim=True)
    s = p * t
    # off before the rounding: the exponent's argument, and t's two sums
    arg = FINE * (abs(scale) * (q.abs() @ k.abs().T) + lse.abs()[:, None]) + FINE
    ps, ss = p * arg, s.abs() * arg + p * FINE * (d_o.abs() @ v.abs().T + (d_o * o).abs().sum(1, keepdim=True))
    ps, ss = ps + LEAST, ss + LEAST * (1 + t.abs())

    def product(w, slack, x):  # w^T x
        terms = torch.minimum(w.abs().T @ x.abs(), 6 * torch.sqrt((w * w).T @ (x * x)))
        return w.T @ x, HALF * terms + slack.T @ x.abs() + FINE * (w.abs().T @ x.abs())

    dv, e_v = product(p, ps * (1 + HALF), d_o)
    dk, e_k = product(s, ss * (1 + HALF), q)
    # dq may be formed of the keys less a vector m within their own range, the mean of some (the sum of S less its rounded values'
    # is known in 32 bits and goes back to m): |k - m| then is |k| and the largest |k| of the channel at most
    dq, e_q = product(s.T, ss.T * (1 + HALF), k.abs() + k.abs().amax(0))
    dq = s @ k
    got = [scale * dq, scale * dk, dv]
    off = [abs(scale) * e_q, abs(scale) * e_k, e_v]
    return got, [HALF * x.abs() + (1 + HALF) * e + LEAST for x, e in zip(got, off)]


def segments(cu_q, cu_k):
    return [(cu_q[i], cu_q[i + 1], cu_k[i], cu_k[i + 1]) for i in range(len(cu_q) - 1)]


def packed_attn(q, k, v, cu_q, cu_k, scale):
    o, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=q.dtype, device=q.device)
    for a, b, c, e in segments(cu_q, cu_k):
        for h in range(q.shape[1]):
            o[a:b, h], lse[a:b, h] = attn(q[a:b, h], k[c:e, h], v[c:e, h], scale)
    return o, lse


def packed_attn_bwd(d_o, q, k, v, o, lse, cu_q, cu_k, scale):
    """[dq, dk, dv] and their tolerances; rows of no segment are 0."""
    got, tol = [torch.zeros_like(x) for x in (q, k, v)], [torch.zeros_like(x) for x in (q, k, v)]
    for a, b, c, e in segments(cu_q, cu_k):
        for h in range(q.shape[1]):
            g, f = attn_bwd(d_o[a:b, h], q[a:b, h], k[c:e, h], v[c:e, h], o[a:b, h], lse[a:b, h], scale)
            for i, (lo, hi) in enumerate(((a, b), (c, e), (c, e))):
                got[i][lo:hi, h], tol[i][lo:hi, h] = g[i], f[i]
    return got, tol


def offsets(lens):
    return [int(x) for x in np.concatenate([[0], np.cumsum(lens)])]
