"""tests/block_ref.py against automatic differentiation in 64 bits and against differences (CPU)."""
import math

import pytest
import torch

import block_ref as R

AXES = {64: (12, 10, 10), 128: (22, 21, 21)}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rand(g, *shape):
    return torch.randn(shape, generator=g, dtype=torch.float64)


def close(a, b, tol=1e-10):
    assert torch.allclose(a, b, rtol=tol, atol=tol), (a - b).abs().max()


@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("d", [64, 128])
def test_rope_is_a_rotation_and_its_gradient_is_autograd_s(d, norm, interleaved):
    g = gen(1)
    x, w, dy = rand(g, 5, 3, d) * 2, 1 + 0.3 * rand(g, d), rand(g, 5, 3, d)
    pos = torch.randint(-1000, 1000, (5, 3), generator=g).int()
    freq = torch.rand(d // 2, generator=g, dtype=torch.float64)
    angle = R.angles(pos, freq, AXES[d])
    assert angle[2, 0] == pos[2, 0] * freq[0] and angle[2, AXES[d][0]] == pos[2, 1] * freq[AXES[d][0]] and angle[3, -1] == pos[3, 2] * freq[-1]
    weight = w if norm else None
    leaves = [x.requires_grad_()] + ([w.requires_grad_()] if norm else [])
    y = R.rope(x, weight, angle, interleaved, 1e-6)
    want = torch.autograd.grad(y, leaves, dy)
    dx, dw, mag, mag_w = R.rope_bwd(dy, x.detach(), None if weight is None else w.detach(), angle, interleaved, 1e-6)
    close(dx, want[0])
    assert bool((mag >= dx.abs() - 1e-12).all())
    if norm:
        close(dw, want[1])
        assert bool((mag_w >= dw.abs() - 1e-12).all())
    else:  # lengths stay, and the pairs are the two orders'
        close(y.square().sum(-1), x.square().sum(-1))
        i = 7
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + d // 2)
        close(torch.complex(y[..., a], y[..., b]),
              torch.complex(x[..., a], x[..., b]) * torch.polar(torch.ones(5, 1, dtype=torch.float64), angle[:, i:i + 1]))


def test_rope_by_differences():
    g = gen(2)
    d, h = 64, 1e-5
    x, w, dy = rand(g, 2, 1, d), 1 + 0.3 * rand(g, d), rand(g, 2, 1, d)
    angle = rand(g, 2, d // 2) * 3
    dx, dw, _, _ = R.rope_bwd(dy, x, w, angle, True, 1e-6)
    for i in (0, 1, 33, 63):
        e = torch.zeros(d, dtype=torch.float64)
        e[i] = h
        for t in range(2):
            at = torch.zeros_like(x)
            at[t, 0] = e
            num = ((R.rope(x + at, w, angle, True, 1e-6) - R.rope(x - at, w, angle, True, 1e-6)) * dy).sum() / (2 * h)
            assert abs(num - dx[t, 0, i]) < 1e-7
        num = ((R.rope(x, w + e, angle, True, 1e-6) - R.rope(x, w - e, angle, True, 1e-6)) * dy).sum() / (2 * h)
        assert abs(num - dw[i]) < 1e-7


@pytest.mark.parametrize("scale", [0.125, -0.3, 0.0])
@pytest.mark.parametrize("m,n", [(1, 1), (1, 7), (5, 1), (9, 13)])
def test_attention_gradients_are_autograd_s(m, n, scale):
    g = gen(3)
    q, k, v, d_o = rand(g, m, 8), rand(g, n, 8), rand(g, n, 8), rand(g, m, 8)
    for x in (q, k, v):
        x.requires_grad_()
    o, lse = R.attn(q, k, v, scale)
    want = torch.autograd.grad(o, (q, k, v), d_o, allow_unused=True)
    got, tol = R.attn_bwd(d_o, q.detach(), k.detach(), v.detach(), o.detach(), lse.detach(), scale)
    for a, b, t in zip(got, want, tol):
        close(a, torch.zeros_like(a) if b is None else b)
        assert bool((t >= 0).all())


def test_attention_gradients_by_differences():
    g = gen(4)
    q, k, v, d_o = (rand(g, n, 6) for n in (4, 5, 5, 4))
    o, lse = R.attn(q, k, v, 0.4)
    got, _ = R.attn_bwd(d_o, q, k, v, o, lse, 0.4)
    h = 1e-5
    for i, x in enumerate((q, k, v)):
        for at in ((0, 0), (3, 5), (2, 1)):
            e = torch.zeros_like(x)
            e[at] = h
            up, down = ([y + e if y is x else y for y in (q, k, v)], [y - e if y is x else y for y in (q, k, v)])
            num = ((R.attn(*up, 0.4)[0] - R.attn(*down, 0.4)[0]) * d_o).sum() / (2 * h)
            assert abs(num - got[i][at]) < 1e-7


def test_segments_without_keys_or_queries():
    g = gen(5)
    cu_q, cu_k = R.offsets([3, 0, 2]), R.offsets([0, 4, 5])
    q, d_o, k, v = rand(g, 5, 2, 8), rand(g, 5, 2, 8), rand(g, 9, 2, 8), rand(g, 9, 2, 8)
    o, lse = R.packed_attn(q, k, v, cu_q, cu_k, 0.3)
    assert bool((o[:3] == 0).all()) and bool((lse[:3] == -math.inf).all())
    (dq, dk, dv), _ = R.packed_attn_bwd(d_o, q, k, v, o, lse, cu_q, cu_k, 0.3)
    assert bool((dq[:3] == 0).all()) and bool((dk[:4] == 0).all()) and bool((dv[:4] == 0).all())
    assert bool((dq[3:] != 0).any()) and bool((dk[4:] != 0).any())


def test_tolerances_hold_for_the_roundings_they_stand_for():
    """P and S rounded to bfloat16, and the results once more, as the kernels do it, in 64 bits otherwise."""
    g = gen(6)
    q, k, v, d_o = (rand(g, n, 64).bfloat16().double() for n in (200, 300, 300, 200))
    k = (k + 2 * rand(g, 64)).bfloat16().double()
    o, lse = R.attn(q, k, v, 0.125)
    got, tol = R.attn_bwd(d_o, q, k, v, o, lse, 0.125)
    p = torch.exp(0.125 * (q @ k.T) - lse[:, None])
    s = p * (d_o @ v.T - (d_o * o).sum(1, keepdim=True))
    p, s = p.bfloat16().double(), s.bfloat16().double()
    for a, b, t in zip((0.125 * (s @ k), 0.125 * (s.T @ q), p.T @ d_o), got, tol):
        off = (a.bfloat16().double() - b).abs()
        assert bool((off <= t).all()) and (off / t).max() > 0.05  # (and they are not idle)
