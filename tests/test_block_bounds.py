"""tests/block_bounds.py on the CPU: the roundings that the kernels make stay within its bounds, mistakes do not."""
import pytest
import torch

import block_bounds as B
import block_ref as R


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rand(g, *shape):
    return torch.randn(shape, generator=g, dtype=torch.float64)


def bf16(x):
    return x.bfloat16().double()


def significant(x, bits):
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(m * 2.0 ** bits), e - bits)


def two(s):
    """S of dq: its rounded value and the rounded rest."""
    return bf16(s) + bf16(s - bf16(s))


def less(mean):
    """S rounded once, and the sum of what that leaves times a mean of keys taken off."""
    return lambda s, k: bf16(s) @ k - (bf16(s) - s).sum(1, keepdim=True) * mean(k)


def rounded(d_o, q, k, v, o, lse, scale, D=1.0, P=1.0, S=bf16, dq=lambda s, k: two(s) @ k):
    """dq, dk, dv of one segment and head with the kernels' roundings, and what may be wrong in them: factors of D and of P, another
    rounding of S for dk, another product for dq."""
    p = P * torch.exp(scale * (q @ k.T) - lse[:, None])
    s = p * (d_o @ v.T - D * (d_o * o).sum(1, keepdim=True))
    return [bf16(scale * dq(s, k)), bf16(scale * (S(s).T @ q)), bf16(bf16(p).T @ d_o)]


def case(name, m, n, d):
    g = gen(7)
    q, v, d_o = (bf16(rand(g, x, d)) for x in (m, n, m))
    k = rand(g, n, d)
    if name == "common":  # channels that stand far out, all to one side
        k, q = k + 8 * rand(g, d).sign(), bf16(0.3 * q)
    elif name == "offset":
        k = k + rand(g, d)
    elif name == "first":  # keys that stand apart and have no weight
        u = rand(g, d).sign()
        k[:32] += 16 * u
        q = 0.3 * q
        q = bf16(q - (q @ u)[:, None] * u / d - 1.2 / d ** 0.5 * u)
    elif name == "hidden":  # a channel that hides all keys but three
        q[:, 3], at = -1, k[[5, n // 2, n - 1], 3].clone()
        k[:, 3] = 30000
        k[[5, n // 2, n - 1], 3] = at
    k = bf16(k)
    scale = d ** -0.5
    o, lse = R.attn(q, k, v, scale)
    return d_o, q, k, v, bf16(o), lse.float().double(), scale


def outside(name, x, **wrong):
    """Which of dq, dk, dv of the kernels' roundings are outside their bounds."""
    want = B.packed(*(y[:, None] for y in x[:6]), [0, x[0].shape[0]], [0, x[2].shape[0]], x[6])
    bad = []
    for what, got, (ref, tol, most) in zip(("dq", "dk", "dv"), rounded(*x, **wrong), want):
        try:
            B.check(what, got[:, None], ref, tol, most)
        except AssertionError:
            bad.append(what)
    return bad


NAMES = ["plain", "offset", "common", "first", "hidden"]
SIZES = [(1, 1), (1, 200), (200, 1), (64, 40), (300, 700)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m,n", SIZES)
def test_what_the_kernels_round_is_within_the_bounds(m, n, d):
    for name in NAMES if n > 32 else NAMES[:2]:
        assert outside(name, case(name, m, n, d)) == [], name


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("name", ["plain", "offset", "common"])
def test_mistakes_are_not(name, d):
    x = case(name, 300, 700, d)
    assert outside(name, x, P=0.99) == ["dq", "dk", "dv"]
    assert outside(name, x, S=lambda s: significant(s, 6)) == ["dk"]
    assert outside(name, x, dq=lambda s, k: bf16(s) @ k) == ["dq"]
    if name != "plain":  # (of many keys without a mean D's part is next to nothing)
        assert outside(name, x, D=0.99) == ["dq"]
    assert "dq" in outside(name, case(name, 300, 40, d), D=0.99)


@pytest.mark.parametrize("d", [64, 128])
def test_means_in_place_of_the_rest_are_not(d):
    """Of the first keys, or of all: keys without weight put dq off by any amount."""
    for name, mean in (("first", lambda k: k[:32].mean(0)), ("hidden", lambda k: k[:32].mean(0)), ("hidden", lambda k: k.mean(0))):
        assert outside(name, case(name, 300, 700, d), dq=less(mean)) == ["dq"]
