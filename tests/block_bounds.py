"""Sharper bounds of attention's gradients than block_ref's tolerances: of every element of dq by the keys as they are, and of each
gradient as a whole.  64 bits, one segment and one head at a time; used by tests/test_block_bounds.py and tests/test_gpu_block_bounds.py."""
import math

import torch

import block_ref as R


def parts(d_o, q, k, v, o, lse, scale):
    """P and S of the definition, and how far each may be off before it is rounded (as in block_ref.attn_bwd: the exponent's
    argument, the two sums of a residual, and what is below 2^-126)."""
    p = torch.exp(scale * (q @ k.T) - lse[:, None])
    t = d_o @ v.T - (d_o * o).sum(1, keepdim=True)
    arg = R.FINE * (abs(scale) * (q.abs() @ k.abs().T) + lse.abs()[:, None]) + R.FINE
    off_p = p * arg + R.LEAST
    off_s = (p * t).abs() * arg + p * R.FINE * (d_o.abs() @ v.abs().T + (d_o * o).abs().sum(1, keepdim=True)) + R.LEAST * (1 + t.abs())
    return p, p * t, off_p, off_s


def common_part(k):
    """Of each channel: the middle of the keys nearest to and furthest from 0, twice the nearest at most; 0 where signs are mixed."""
    near, far = k.abs().amin(0), k.abs().amax(0)
    m = torch.minimum((near + far) / 2, 2 * near)
    return torch.where((k > 0).all(0), m, torch.where((k < 0).all(0), -m, 0 * m))


def beside_common_part(k, splits, part=common_part):
    """|k - m| with the m of each key's range, of `splits` of them in steps of 64 keys."""
    steps, out = (k.shape[0] + 63) // 64, k.clone()
    for i in range(splits):
        a, b = steps * i // splits * 64, min(steps * (i + 1) // splits * 64, k.shape[0])
        if a < b:
            out[a:b] -= part(k[a:b])
    return out.abs()


def dq_tolerance(dq, s, off_s, k, scale, splits):
    """How far each element of dq = scale S k may be off.  Rounding S gives an error e_j <= HALF |S_j|, one way or the other.  The kernels
    take (sum_j e_j) m off the result, with an m of each channel and range for which |k_j - m| <= |k_j| for every key j: what
    is left is sum_j e_j (k_j - m), HALF sum |S_j (k_j - m)| at the very most and 6 sqrt(sum (S_j (k_j - m))^2) HALF in one of 10^7
    cases; where the ranges are the library's (splits 0), |k_j| stands for |k_j - m|.  The two sums whose difference
    is taken are in 32 bits, FINE sum |S_j| each at most, and |m| <= 2 |k_j|: 4 FINE sum |S_j k_j|, beside the product's own FINE
    sum |S_j k_j|."""
    size, far = s.abs() @ k.abs(), beside_common_part(k, splits)
    terms = torch.minimum(s.abs() @ far, 6 * torch.sqrt((s * s) @ (far * far)))
    e = abs(scale) * (R.HALF * terms + (1 + R.HALF) * (off_s @ k.abs()) + 5 * R.FINE * size)
    return R.HALF * dq.abs() + (1 + R.HALF) * e + R.LEAST


def off_at_most(x, w, off_w, y, scale=1.0, far=None):
    """The norm that the error of x = scale w y has at most.  A rounding to bfloat16 is uniform within half a step, HALF of the value at
    most: a variance of HALF^2 / 3 of the value's square at most, of each weight w (times y, or `far`) and of each result, and
    none goes by another.  What the weights are off before counts in full.  The sum of squares is off from its mean by a share that
    falls with the rows, among which nothing is shared: 4 deviations of sqrt(2 / rows) each."""
    far = y if far is None else far
    var = (R.HALF ** 2 / 3 * (x * x + scale * scale * ((w * w) @ (far * far))) + scale * scale * ((off_w * off_w) @ (y * y))).sum()
    return math.sqrt(var * (1 + 4 * math.sqrt(2 / max(x.shape[0], 1))))


def check(name, got, ref, tol, most, say=lambda *a: None):
    """One gradient of all segments and heads: got [rows, H, d] against ref, elements by tol and the whole by most (norms of each
    segment's and head's error, to be joined)."""
    off = (got.double() - ref).abs()
    bad = ~(off <= tol)
    norm, bound = off.norm().item(), math.sqrt(sum(m * m for m in most))
    say(name, "worst %.3f of its tolerance, norm of the error %.3g of %.3g, %.3f of its bound" % (
        (off / tol.clamp(min=1e-300)).max().item() if off.numel() else 0.0, norm, ref.norm().item(), norm / max(bound, 1e-300)))
    assert not bad.any(), "%s: %d of %d elements off, first at %s: %r for %r, tolerance %r" % (
        name, bad.sum().item(), bad.numel(), bad.nonzero()[0].tolist(), got[bad][0].item(), ref[bad][0].item(), tol[bad][0].item())
    assert norm <= bound, "%s: off by %.3g in all, %.3g at most" % (name, norm, bound)


def packed(d_o, q, k, v, o, lse, cu_q, cu_k, scale, splits=0):
    """[(gradient, its tolerance, its norms' bounds)] of dq, dk and dv; rows of segments without the other side are 0, exactly."""
    out = [[torch.zeros_like(x), torch.zeros_like(x), []] for x in (q, k, v)]
    for a, b, c, e in R.segments(cu_q, cu_k):
        if a == b or c == e:
            continue
        for h in range(q.shape[1]):
            x = d_o[a:b, h], q[a:b, h], k[c:e, h], v[c:e, h], o[a:b, h], lse[a:b, h]
            p, s, off_p, off_s = parts(*x, scale)
            g, tol = R.attn_bwd(*x, scale)
            tol[0] = dq_tolerance(g[0], s, off_s, x[2], scale, splits)
            most = (off_at_most(g[0], s, off_s, x[2], scale, beside_common_part(x[2], splits)), off_at_most(g[1], s.T, off_s.T, x[1], scale),
                    off_at_most(g[2], p.T, off_p.T, x[0]))
            for i, (lo, hi) in enumerate(((a, b), (c, e), (c, e))):
                out[i][0][lo:hi, h], out[i][1][lo:hi, h] = g[i], tol[i]
                out[i][2].append(most[i])
    return out
