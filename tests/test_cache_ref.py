"""Pins of the session cache's reference (cache_ref.py) on the CPU: its e4m3 against torch's type, its exponents against the
definition, its attention against torch's in 64 bits, its eviction against a hand-made case."""
import math

import numpy as np
import torch

import cache_ref as R


def test_e4m3_values_and_rounding_are_torch_s():
    every = torch.arange(256, dtype=torch.uint8)
    np.testing.assert_array_equal(every.view(torch.float8_e4m3fn).double().numpy(), R.VALUES)
    g = torch.Generator().manual_seed(0)
    mids = (R.VALUES[:126] + R.VALUES[1:127]) / 2
    x = np.concatenate([R.VALUES[:127], -R.VALUES[:127], mids, -mids, np.nextafter(mids, 0), np.nextafter(mids, 500),
                        (torch.randn(20000, generator=g, dtype=torch.float64) * torch.exp2(4 * torch.randn(20000, generator=g, dtype=torch.float64)))
                        .clamp(-448, 448).float().double().numpy()])
    x = x.astype(np.float32).astype(np.float64)  # torch rounds from float32
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(R.round_e4m3(x), want)
    assert np.all(R.round_e4m3(np.array([math.inf, -math.inf, math.nan])) & 127 == 127)


def test_exponent_is_the_least_that_fits():
    for top in (448.0, 449.0, 1.0, 0.875, 0.876, 3.5, 7.0, 2.0 ** 60, 2.0 ** -90, 1e-20):
        n = R.exponent([0.1 * top, -top, math.inf, math.nan]) - 127
        assert top <= 448 * 2.0 ** n and top > 448 * 2.0 ** (n - 1)
    assert R.exponent([0.0]) == R.exponent([]) == R.exponent([2.0 ** -130]) == 27


def pool(seed, pages=6, H=2, d=64):
    r = np.random.RandomState(seed)
    return R.Pool(r.randint(0, 126, (pages, H, 64, d)).astype(np.uint8) | (r.randint(0, 2, (pages, H, 64, d)).astype(np.uint8) << 7),
                  r.randint(0, 126, (pages, H, 64, d)).astype(np.uint8), r.randint(120, 123, (pages, H)).astype(np.uint8),
                  r.randint(120, 123, (pages, H)).astype(np.uint8), r.rand(pages, H, 64).astype(np.float32))


def test_attend_and_weigh_are_softmax():
    p = pool(1)
    table, lens, cu = [[4, 1, 0], [2, 3, 5]], [130, 70], [0, 3, 5]
    q = np.random.RandomState(2).randn(5, 4, 64)
    o, lse, _ = R.attend(p, q, cu, table, lens, 0.01)
    got = R.weigh(p, q, lse, cu, table, lens, 0.01) - p.weight
    for s in range(2):
        for hq in range(4):
            k, v = (torch.from_numpy(p.tokens(n, table[s], lens[s], hq // 2)) for n in ("k", "v"))
            x = torch.from_numpy(q[cu[s]:cu[s + 1], hq])
            want = torch.nn.functional.scaled_dot_product_attention(x[None], k[None], v[None], scale=0.01)[0]
            np.testing.assert_allclose(o[cu[s]:cu[s + 1], hq], want.numpy(), rtol=1e-9, atol=1e-9)
        rows = (cu[s + 1] - cu[s]) * 2  # each query row and head of a group hands out one
        for h in range(2):
            total = sum(got[table[s][j // 64], h, j % 64] for j in range(lens[s]))
            assert abs(total - rows) < 1e-6


def test_append_then_evict_by_hand():
    p = R.Pool(*(np.zeros(s, t) for s, t in (((3, 1, 64, 64), np.uint8), ((3, 1, 64, 64), np.uint8), ((3, 1), np.uint8), ((3, 1), np.uint8),
                                            ((3, 1, 64), np.float32))))
    x = np.zeros((5, 1, 64))
    x[:, 0, 0] = [1, 2, 448, 900, 3]  # 900 needs n = 2; 1, 2 and 3 are multiples of 2^2 2^-9
    assert R.append(p, x, x, [0, 5], [[2]], [0], 1) == [5]
    assert p.k_exp[2, 0] == 129 and [float(v) for v in p.tokens("k", [2], 5, 0)[:, 0]] == [1, 2, 448, 896, 3]
    p.weight[2, 0, :5] = [5, 1, 1, 9, 0]
    lens, kept = R.evict(p, [[2]], [5], [[0]], 3, 1, 0)
    assert lens == [3] and kept.tolist() == [[[0, 1, 3]]]
    assert [float(v) for v in p.tokens("v", [0], 3, 0)[:, 0]] == [1, 2, 896] and p.weight[0, 0, :3].tolist() == [5, 1, 9]
