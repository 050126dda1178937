"""Sharper bounds of attention's gradients than block_ref's tolerances: of every element of dq by S in two parts, and of each gradient
as a whole.  64 bits, one segment and one head at a time; used by tests/test_block_bounds.py and tests/test_gpu_block_bounds.py."""
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


def dq_tolerance(dq, s, off_s, k, scale):
    """How far each element of dq = scale S k may be off.  S is taken in two parts, its rounded value and the rounded rest, which leaves
    HALF^2 |S_j| of each at most, one way or the other: HALF^2 sum |S_j k_j| at the very most, 6 sqrt(sum (S_j k_j)^2) HALF^2 in one of
    10^7 cases; the product's sum is in 32 bits."""
    size = s.abs() @ k.abs()
    terms = torch.minimum(size, 6 * torch.sqrt((s * s) @ (k * k)))
    e = abs(scale) * (R.HALF ** 2 * terms + (1 + R.HALF) * (off_s @ k.abs()) + R.FINE * size)
    return R.HALF * dq.abs() + (1 + R.HALF) * e + R.LEAST


def half_step(x):
    """Of the bfloat16 values around x: HALF of the power of two below it."""
    return torch.ldexp(torch.full_like(x, R.HALF / 2), torch.frexp(x)[1]) * (x != 0)


def off_at_most(x, w, off_w, y, scale=1.0, parts=1):
    """The norm that the error of x = scale w y has at most.  A rounding to bfloat16 is uniform within half a step, a variance of a third of
    its square, of each weight w (of its rest, where w is taken in two parts) and of each result, and none goes by another.
    What the weights are off before counts in full.  So a row's squares have a mean v_r, and deviate from it by sqrt(2) v_r at most (all of
    one row's in step); the rows share no weight, so their sum deviates by sqrt(2 sum v_r^2), of which 4 are allowed for.  (That is the sum's
    sqrt(2 / rows) where the rows are alike, and more where few rows have most of it.)"""
    of_w = half_step(w) * (1 if parts == 1 else R.HALF)
    v = (half_step(x).square() / 3 + scale * scale * ((of_w.square() / 3 + off_w.square()) @ y.square())).sum(1)
    return math.sqrt(v.sum() + 4 * math.sqrt(2 * v.square().sum()))


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


def packed(d_o, q, k, v, o, lse, cu_q, cu_k, scale):
    """[(gradient, its tolerance, its norms' bounds)] of dq, dk and dv; rows of segments without the other side are 0, exactly."""
    out = [[torch.zeros_like(x), torch.zeros_like(x), []] for x in (q, k, v)]
    for a, b, c, e in R.segments(cu_q, cu_k):
        if a == b or c == e:
            continue
        for h in range(q.shape[1]):
            x = d_o[a:b, h], q[a:b, h], k[c:e, h], v[c:e, h], o[a:b, h], lse[a:b, h]
            p, s, off_p, off_s = parts(*x, scale)
            g, tol = R.attn_bwd(*x, scale)
            tol[0] = dq_tolerance(g[0], s, off_s, x[2], scale)
            most = (off_at_most(g[0], s, off_s, x[2], scale, parts=2), off_at_most(g[1], s.T, off_s.T, x[1], scale),
                    off_at_most(g[2], p.T, off_p.T, x[0]))
            for i, (lo, hi) in enumerate(((a, b), (c, e), (c, e))):
                out[i][0][lo:hi, h], out[i][1][lo:hi, h] = g[i], tol[i]
                out[i][2].append(most[i])
    return out
