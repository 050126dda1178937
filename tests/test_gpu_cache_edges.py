"""The 8-bit session cache on the GPU where its calls are easiest to get wrong: sessions whose offsets contradict each
other, rows that one key dominates, the log-sum-exp's last bits, the ends of the number formats, what is not finite, and
work that is dealt out in equal shares."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import cache_ref as R

pytestmark = pytest.mark.gpu

ts = pytest.importorskip("paper_2606_19271_amd")

PAGE = 64
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ts.load_cache()
    return torch.device("cuda:0")


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def filled(g, lens, H, d, k=1.0, v=1.0, spare=0):
    """A pool that holds sessions of these lengths, appended in one call, and their table."""
    need = [-(-n // PAGE) for n in lens]
    width = max(need + [1])
    order = torch.randperm(sum(need) + spare, generator=g, device="cuda").tolist()
    cache = ts.session_cache(max(1, sum(need) + spare), H, d)
    table = [[order.pop() for _ in range(n)] + [-1] * (width - n) for n in need]
    cu = [0] + np.cumsum(lens).tolist()
    k = (normal(g, cu[-1], H, d) * k).bfloat16() if not torch.is_tensor(k) else k
    v = (normal(g, cu[-1], H, d) * v).bfloat16() if not torch.is_tensor(v) else v
    ts.ts_cache_append(cache, k, v, ints(cu), max(lens + [1]), ints(table), ints([0] * len(lens)))
    return cache, table


def same(a, b):
    return all(torch.equal(x.view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32), y.view(
        torch.int16 if y.dtype == torch.bfloat16 else torch.int32)) for x, y in zip(a, b))


# ---- offsets that contradict each other

# (offsets, most rows): a backward session is skipped, and those after it name rows that earlier ones have
OVERLAPS = [([0, 1000, 0, 1000, 0, 1000, 2000], 1000), ([0, 1000, 0, 3000, 4000], 3000), ([0, 1000] * 35 + [2000], 1000)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("splits", [0, 1, 3])
@pytest.mark.parametrize("cu,most", OVERLAPS)
def test_attn_sessions_that_overlap_leave_the_others_alone(cu, most, splits, d):
    """More row tiles than disjoint sessions could have: the last session, the shortest and of rows that nobody else
    names, gets the result that it gets alone."""
    g = gen(len(cu) + splits + d)
    H, n = 12, len(cu) - 1
    lens = [200] * (n - 1) + [90]
    cache, table = filled(g, lens, H, d)
    q = normal(g, cu[-1], H, d).bfloat16()
    out, lse = torch.full_like(q, 7.0), torch.full((cu[-1], H), 7.0, device="cuda")
    ts.ts_cache_attn(q, cache, ints(cu), most, ints(table), ints(lens), 256, out=out, lse=lse, num_splits=splits)
    rows = slice(cu[-2], cu[-1])
    alone = ts.ts_cache_attn(q[rows].contiguous(), cache, ints([0, cu[-1] - cu[-2]]), most, ints(table[-1:]), ints(lens[-1:]), 256,
                             return_lse=True, num_splits=max(splits, 1))
    # two results, each off by a rounding of the weights and one of the result: 2^-8 of an average of the values' sizes each
    assert (out[rows].float() - alone[0].float()).abs().max() <= 4 * 2.0 ** -8 * 6
    assert (lse[rows] - alone[1]).abs().max() <= 1e-4
    assert torch.all(out[:cu[-2]] != 7.0)


# ---- the log-sum-exp's last bits

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [20, 70])
def test_lse_of_equal_scores(rows, d):
    """Queries of zeros: every weight is the same power of two and every sum exact, so that the log-sum-exp is ln of the
    length but for one logarithm (an ulp, 2^-23), the constant ln 2 (2^-25) and their product's rounding (2^-24): less than
    2^-22 of its value."""
    lens = [1, 2, 3, 5, 17, 63, 64, 65, 100, 127, 128, 129, 200, 333, 500, 700, 1000, 1023, 1300, 1999]
    g = gen(rows + d)
    cache, table = filled(g, lens, 1, d)
    q = torch.zeros(rows * len(lens), 1, d, dtype=torch.bfloat16, device="cuda")
    cu = [rows * i for i in range(len(lens) + 1)]
    _, lse = ts.ts_cache_attn(q, cache, ints(cu), rows, ints(table), ints(lens), max(lens), return_lse=True, num_splits=1)
    got = lse.double().cpu().numpy().reshape(len(lens), rows)
    want = np.log(lens)[:, None]
    assert np.all(np.abs(got - want) <= 2.0 ** -22 * want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [20, 70])
def test_lse_of_one_token(rows, d):
    """One key: the log-sum-exp is its score.  q and k have one channel that is not zero and few bits, so the product is
    exact; scaled to log2 units (2^-23: the constant and a rounding), taken from the running maximum and put back (a weight's
    exponent is good to 2^-21, half a step at the size of the bias), and times ln 2 (2^-23)."""
    n = 50
    score = torch.arange(1, n + 1).float() * 0.375 - 9.0
    k = torch.zeros(n, 1, d)
    k[:, 0, 0] = score
    k = k.bfloat16().cuda()
    cache, table = filled(gen(1), [1] * n, 1, d, k=k, v=k)
    q = torch.zeros(n * rows, 1, d, dtype=torch.bfloat16, device="cuda")
    q[:, 0, 0] = 1.0
    pool = R.Pool.of(cache)
    want = np.array([pool.tokens("k", table[s], 1, 0)[0, 0] for s in range(n)])[:, None]
    _, lse = ts.ts_cache_attn(q, cache, ints([rows * i for i in range(n + 1)]), rows, ints(table), ints([1] * n), 64, scale=1.0,
                              return_lse=True, num_splits=1)
    got = lse.double().cpu().numpy().reshape(n, rows)
    assert np.all(np.abs(got - want) <= 2.0 ** -21 * math.log(2) + 2.0 ** -22 * np.abs(want))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,splits", [(3, 1), (70, 1), (70, 3)])
@pytest.mark.parametrize("size", [-96, -104])
def test_attn_of_the_smallest_values(size, rows, splits, d):
    """Values near the least exponent of a page: products with weights of 2^-15 of the largest one's size stay normal numbers.
    The weights' rounding (2^-8 of the values' average size), the result's (2^-8), a score good to (d + 2) 2^-24 of its terms' sum, and
    what a product under 2^-126 could lose: n weights of less than 2^-111 / |v|, relative to a total of at least 1."""
    g = gen(rows + d + splits)
    H, n = 2, 400
    cache, table = filled(g, [n], H, d, v=2.0 ** size)
    q = normal(g, rows, H, d).bfloat16()
    o = ts.ts_cache_attn(q, cache, ints([0, rows]), rows, ints(table), ints([n]), n, num_splits=splits)
    pool, q64 = R.Pool.of(cache), q.double().cpu().numpy()
    scale = float(np.float32(1 / math.sqrt(d)))
    ro, _, av = R.attend(pool, q64, [0, rows], table, [n], scale)
    terms = max(np.abs(pool.tokens("k", table[0], n, h)).max() for h in range(H)) * np.abs(q64).sum(2).max() * scale
    bound = (2.0 ** -8 + 2 * (d + 2) * 2.0 ** -24 * terms) * av + 2.0 ** -8 * np.abs(ro) + n * 2.0 ** -133
    off = np.abs(o.double().cpu().numpy() - ro)
    assert np.all(off <= bound), (off / bound).max()


# ---- rows that one key dominates

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,G,rows,n,splits", [(1, 1, 300, 1300, 1), (2, 2, 70, 1999, 1), (1, 1, 300, 3000, 4), (1, 1, 513, 777, 0)])
@pytest.mark.parametrize("gain", [0.5, 2.0, 5.0])
def test_attn_of_equal_values(gain, H, G, rows, n, splits, d):
    """Values that are the same for every token, so that whatever the weights O is that value, but for their rounding to 16 bits:
    2^-8 of it at most, and a rounding of the result.  A key that holds more than 16/17 of a row is more than 16 times what
    comes before it, and its weight is exact: there only the others' seventeenth is off, by less than the 0.53 * 2^-8 that half a
    step is of these values (mantissas up to 1.875), and O is the value itself."""
    g = gen(rows + n + d)
    v = torch.tensor([1.875, -1.75, 3.5, 0.9375])[torch.arange(d) % 4].expand(n, H, d).bfloat16().contiguous().cuda()
    cache, table = filled(g, [n], H, d, k=gain, v=v)
    q = normal(g, rows, H * G, d).bfloat16()
    args = (q, cache, ints([0, rows]), rows, ints(table), ints([n]), n)
    o, _ = ts.ts_cache_attn(*args, return_lse=True, num_splits=splits)
    assert torch.equal(ts.ts_cache_attn(*args, num_splits=splits), o)
    pool, held = R.Pool.of(cache), torch.zeros(rows, H * G, dtype=torch.bool, device="cuda")
    for hq in range(H * G):
        k = torch.from_numpy(pool.tokens("k", table[0], n, hq // G)).cuda()
        w = torch.softmax(q[:, hq].double() @ k.T / math.sqrt(d), 1)
        held[:, hq] = w.max(1).values > 0.945
    assert held.any() or gain < 5
    want = v[:1, :1].expand_as(o)
    assert torch.equal(o[held], want[held])
    assert ((o.double() / want.double()) - 1).abs().max() <= 2 * 2.0 ** -8


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("height", [4.3, 4.9, 7.9])
def test_attn_of_a_dominating_key(height, d):
    """One key of more than 16 times the weight of all that come before it, in a tile between the first and the last, and of values where
    the others have zeros: O is the key's value times its share, within a rounding of the result (2^-8) and the shift of two
    scores (each good to (d + 2) 2^-24 of its one term, 10 at most here, and 2^-20).  Had its weight been rounded too, it would be
    off by up to another 2^-8."""
    n, rows, at = 400, 80, 200
    k, v = torch.zeros(n, 1, d), torch.zeros(n, 1, d)
    k[:, 0, 0] = -4.0
    k[at, 0, 0] = 4.0
    v[at, 0] = torch.tensor([1.875, -1.25, 3.5, 1.0])[torch.arange(d) % 4]
    cache, table = filled(gen(2), [n], 1, d, k=k.bfloat16().cuda(), v=v.bfloat16().cuda())
    q = torch.zeros(rows, 1, d)
    q[:, 0, 0] = height * (1 + torch.arange(rows) / rows / 8)
    q = q.bfloat16().cuda()
    o = ts.ts_cache_attn(q, cache, ints([0, rows]), rows, ints(table), ints([n]), n, scale=0.25, num_splits=1).double().cpu().numpy()
    ro, _, _ = R.attend(R.Pool.of(cache), q.double().cpu().numpy(), [0, rows], table, [n], 0.25)
    assert np.all(np.abs(o - ro) <= (2.0 ** -8 + 2 * (d + 2) * 2.0 ** -24 * 20 + 2.0 ** -19) * np.abs(ro))


# ---- the ends of the format

def test_append_and_evict_of_the_largest_magnitudes():
    """The largest bfloat16 magnitudes would round to 2^128, which no bfloat16 holds: they become the largest element that does,
    240 * 2^120, so that every element is a finite bfloat16 and survives an eviction."""
    d, H = 64, 2
    top = torch.tensor([0x7f00, 0x7f60, 0x7f61, 0x7f70, 0x7f71, 0x7f77, 0x7f78, 0x7f7f], dtype=torch.int16)  # 2^127 .. the largest
    x = torch.zeros(70, H, d, dtype=torch.bfloat16)
    x.view(torch.int16)[:, 0] = top[torch.arange(70 * d) % 8].reshape(70, d)
    x[:, 1] = -x[:, 0]
    x[3, 0, 0], x[4, 0, 0] = math.inf, math.nan
    cache = ts.session_cache(4, H, d)
    x = x.cuda()
    ts.ts_cache_append(cache, x, x, ints([0, 70]), 70, ints([[2, 0]]), ints([0]))
    pool = R.Pool.of(cache)
    assert np.all(pool.k_exp[[2, 0]] == 247) and np.all(pool.v_exp[[2, 0]] == 247)
    xs = x.double().cpu().numpy()
    want = np.minimum(np.abs(np.where(np.isfinite(xs), xs, 0)), 240 * 2.0 ** 120)
    want = R.VALUES[R.round_e4m3(want * 2.0 ** -120)] * 2.0 ** 120 * np.where(np.isfinite(xs), np.sign(np.nan_to_num(xs)), np.nan)
    for name in ("k", "v"):
        for h in range(H):
            got = pool.tokens(name, [2, 0], 70, h)
            np.testing.assert_array_equal(got, want[:, h])
            fine = np.isfinite(got)
            assert np.all(torch.from_numpy(got[fine]).bfloat16().double().numpy() == got[fine])
    # older tokens of a page whose exponent rises, and an eviction
    cache.weight.copy_(torch.rand(cache.weight.shape, generator=gen(1), device="cuda"))
    ts.ts_cache_append(cache, x[:1] * 0.25, x[:1], ints([0, 1]), 1, ints([[2, 0]]), ints([70]))
    want_pool = R.Pool.of(cache)
    ts.ts_cache_evict(cache, ints([[2, 0]]), ints([71]), 71, ints([[1]]), 40, 5, 5)
    R.evict(want_pool, [[2, 0]], [71], [[1]], 40, 5, 5)
    for name in ("k", "v"):
        assert R.same_values(getattr(cache, name).view(torch.uint8).cpu().numpy(), getattr(want_pool, name))
        np.testing.assert_array_equal(getattr(cache, name + "_exp").cpu().numpy(), getattr(want_pool, name + "_exp"))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,n,splits", [(1, 5000, 1), (3, 5000, 0), (40, 900, 3), (300, 5000, 1), (300, 3000, 5)])
def test_attn_of_the_largest_values(rows, n, splits, d):
    """Values of the largest size that a page holds, the same for every token: O is that value, whatever the number of tokens
    whose products are added up on the way to it."""
    v = torch.full((n, 1, d), 240 * 2.0 ** 120)
    v[:, :, 1::2] *= -1
    cache, table = filled(gen(n), [n], 1, d, k=0.1, v=v.bfloat16().cuda())
    q = normal(gen(rows), rows, 1, d).bfloat16()
    o = ts.ts_cache_attn(q, cache, ints([0, rows]), rows, ints(table), ints([n]), n, num_splits=splits)
    want = v[:1].bfloat16().cuda().expand_as(o)
    # sums of up to n weights, each rounded to 2^-8 of itself, over their fp32 sum
    assert torch.isfinite(o).all() and ((o.double() / want.double()) - 1).abs().max() <= 2 * 2.0 ** -8


# ---- a process's first call

FIRST = r"""
import sys; sys.path.insert(0, %r)
import torch
import paper_2606_19271_amd as ts
from paper_2606_19271_amd import _lib
cache = ts.session_cache(40, 2, 64)
cache.k.view(torch.uint8).random_(0, 100); cache.v.view(torch.uint8).random_(0, 100)
cache.k_exp.fill_(120); cache.v_exp.fill_(120)
ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
args = (torch.randn(300, 2, 64, device="cuda").bfloat16(), cache, ints([0, 300]), 300, ints([list(range(40))]), ints([2500]), 2560)
x = torch.zeros(4, device="cuda") + 1
torch.cuda.synchronize()
graph, status = torch.cuda.CUDAGraph(), None
with torch.cuda.graph(graph):
    x.add_(1)
    try:
        ts.ts_cache_attn(*args)
    except ts.TsAttnError as e:
        status = e.status
print("status", status == _lib.TS_ERR_CAPTURE, flush=True)
want = ts.ts_cache_attn(*args)
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    got = ts.ts_cache_attn(*args)
graph.replay()
torch.cuda.synchronize()
print("same", torch.equal(got.view(torch.int16), want.view(torch.int16)), flush=True)
"""


def test_a_process_s_first_call_under_capture_is_refused():
    """And leaves the capture usable; after a call outside capture, one under it is recorded."""
    r = subprocess.run([sys.executable, "-c", FIRST % ROOT], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "status True" in r.stdout and "same True" in r.stdout, r.stdout + r.stderr


# ---- what a session's bits depend on

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [[3, 16, 1], [20, 17, 64], [300, 70, 129]])
@pytest.mark.parametrize("splits", [1, 3])
def test_a_session_s_bits_with_forced_ranges(rows, splits, d):
    """Alone, with its own rows as the most, and in a batch whose most is of the same kind (up to 16, up to 64, more): the same."""
    g = gen(sum(rows) + splits)
    H, lens = 2, [900, 333, 2000]
    cache, table = filled(g, lens, H, d)
    cu = [0] + np.cumsum(rows).tolist()
    q = normal(g, cu[-1], H, d).bfloat16()
    o, lse = ts.ts_cache_attn(q, cache, ints(cu), max(rows), ints(table), ints(lens), 2000, return_lse=True, num_splits=splits)
    for s, n in enumerate(rows):
        r = slice(cu[s], cu[s + 1])
        alone = ts.ts_cache_attn(q[r].contiguous(), cache, ints([0, n]), n, ints(table[s:s + 1]), ints(lens[s:s + 1]), lens[s],
                                 return_lse=True, num_splits=splits)
        assert same(alone, [o[r], lse[r]]), s


@pytest.mark.parametrize("rows", [5, 90])
@pytest.mark.parametrize("scale", [3.4e38, -3.4e38, 1e-45])
def test_scales_at_the_ends_of_float32(scale, rows):
    """Any finite scale: queries of zeros have equal weights for every token, by the formula."""
    d, n = 64, 300
    cache, table = filled(gen(rows), [n], 1, d)
    q = torch.zeros(rows, 1, d, dtype=torch.bfloat16, device="cuda")
    args = (ints([0, rows]), rows, ints(table), ints([n]), n)
    o, lse = ts.ts_cache_attn(q, cache, *args, scale=scale, return_lse=True)
    pool = R.Pool.of(cache)
    v = pool.tokens("v", table[0], n, 0)
    # (weights of equal powers of two: exact; fp32 sums, and a rounding of the result)
    assert np.all(np.abs(o.double().cpu().numpy()[:, 0] - v.mean(0)) <= 2.0 ** -8 * np.abs(v.mean(0)) + 2.0 ** -20 * np.abs(v).mean(0))
    assert (lse.double() - math.log(n)).abs().max() <= 2.0 ** -22 * math.log(n)
    w = ts.ts_cache_weigh(q, lse, cache, *args, scale=scale, out=torch.zeros_like(cache.weight))
    got = torch.cat([w[p, 0] for p in table[0]])[:n]
    assert (got - rows / n).abs().max() <= 1e-5 * rows / n


# ---- what is not finite

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,splits", [(3, 0), (40, 2), (70, 1), (300, 1), (300, 3)])
def test_attn_of_queries_that_are_not_finite(rows, splits, d):
    """A query of NaN or infinities makes its own row NaN and no other: the rows beside it stay within a rounding of the weights
    and one of the result (2^-8 of the values each) of what they are without it."""
    g = gen(rows + d)
    H, n = 2, 900
    cache, table = filled(g, [n], H, d)
    q = normal(g, rows, H, d).bfloat16()
    args = (cache, ints([0, rows]), rows, ints(table), ints([n]), n)
    o, lse = ts.ts_cache_attn(q, *args, return_lse=True, num_splits=splits)
    bad = q.clone()
    bad[0, 0, 3], bad[rows // 2, 1, 0], bad[rows - 1, 0, d - 1] = math.nan, math.inf, -math.inf
    o2, lse2 = ts.ts_cache_attn(bad, *args, return_lse=True, num_splits=splits)
    hit = torch.zeros(rows, H, dtype=torch.bool, device="cuda")
    hit[0, 0] = hit[rows // 2, 1] = hit[rows - 1, 0] = True
    assert torch.isnan(o2[hit]).all() and torch.isnan(lse2[hit]).all()
    assert (o2[~hit].float() - o[~hit].float()).abs().max() <= 4 * 2.0 ** -8 * 6
    assert (lse2[~hit] - lse[~hit]).abs().max() <= 1e-4


# ---- equal shares of the work

def shares_of(rows, lens, H, G, d):
    """The number of equal shares that the library deals this call out in (by its workspace: two slots of 256 rows to a share),
    or 0."""
    total = sum(rows)
    need = ts.load_cache().ts_cache_attn_workspace(len(rows), max(rows), max(lens), total, H, H * G, d, 0)
    for n in range(2, 1025):
        slots = 2 * n * 256 * 4
        if need == slots + 2 * n * 256 * d * 4:
            return n
    return 0


SHARED = dict(H=32, rows=[280, 90, 300, 257], lens=[9000, 2000, 5000, 6001])


@pytest.mark.parametrize("d", [64, 128])
def test_shares_with_bad_sessions_and_pages(d):
    """Sessions that break the rules leave their rows, also between two that are cut; a page outside the pool inside a cut item
    makes its session NaN; the others are what they are alone."""
    g = gen(d)
    H, rows, lens = SHARED["H"], SHARED["rows"] + [70, 0], SHARED["lens"] + [300, 77]
    assert shares_of(rows, lens, H, 1, d) > 1
    cu = [0] + np.cumsum(rows).tolist()
    cache, table = filled(g, lens, H, d, spare=1)
    stated = list(lens)
    stated[1] = 9001  # longer than the most that is stated
    stated[4] = -1
    table[2][40] = 1 << 29
    q = normal(g, cu[-1], H, d).bfloat16()
    out, lse = torch.full_like(q, 7.0), torch.full((cu[-1], H), 7.0, device="cuda")
    ts.ts_cache_attn(q, cache, ints(cu), max(rows), ints(table), ints(stated), 9000, out=out, lse=lse)
    for s, n in enumerate(rows):
        r = slice(cu[s], cu[s + 1])
        if s in (1, 4):
            assert torch.all(out[r] == 7.0) and torch.all(lse[r] == 7.0)
        elif s == 2:
            assert torch.isnan(out[r]).all() and torch.isnan(lse[r]).all()
        elif n:
            o, l = ts.ts_cache_attn(q[r].contiguous(), cache, ints([0, n]), n, ints(table[s:s + 1]), ints(lens[s:s + 1]), lens[s], return_lse=True,
                                    num_splits=1)
            # two results, each off by a rounding of the weights and one of the result: 2^-8 of an average of the values' sizes each
            assert (out[r].float() - o.float()).abs().max() <= 4 * 2.0 ** -8 * 6
            assert (lse[r] - l).abs().max() <= 1e-4


def shared_step(g, d):
    H, rows, lens = SHARED["H"], SHARED["rows"], SHARED["lens"]
    assert shares_of(rows, lens, H, 1, d) > 1
    cache, table = filled(g, lens, H, d)
    cu = [0] + np.cumsum(rows).tolist()
    return normal(g, cu[-1], H, d).bfloat16(), (cache, ints(cu), max(rows), ints(table), ints(lens), max(lens))


@pytest.mark.parametrize("d", [64, 128])
def test_shares_in_a_graph(d):
    g = gen(20 + d)
    q, args = shared_step(g, d)
    ts.ts_cache_attn(q, *args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ts.ts_cache_attn(q, *args, return_lse=True)
    for i in range(4):
        q.copy_(normal(g, *q.shape).bfloat16())
        want = ts.ts_cache_attn(q, *args, return_lse=True)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert same(got, want), i


def test_shares_on_two_streams():
    g = gen(30)
    steps = [shared_step(g, 128), shared_step(g, 64)]
    want = [ts.ts_cache_attn(q, *args, return_lse=True) for q, args in steps]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in steps], []
    for _ in range(4):
        for i, (q, args) in enumerate(steps):
            with torch.cuda.stream(streams[i]):
                got.append((i, ts.ts_cache_attn(q, *args, return_lse=True)))
    torch.cuda.synchronize()
    for i, r in got:
        assert same(r, want[i])


# ---- 33 to 64 rows of a cached head, where large row tiles take fewer and longer ranges of keys

@pytest.mark.parametrize("d,H,G,rows,lens", [(128, 12, 1, [64], [8192]), (128, 6, 2, [20, 32], [8001, 7000]), (64, 12, 1, [64, 1], [8192, 100]),
                                             (64, 24, 1, [40], [8000]), (128, 40, 1, [33], [4095])])
def test_attn_of_up_to_64_rows_in_large_tiles(d, H, G, rows, lens):
    """Against ranges of the row kernel, which forced ones are: two results, each off by a rounding of the weights and one of the
    result, 2^-8 of an average of the values' sizes each."""
    g = gen(d + H + rows[0])
    cache, table = filled(g, lens, H, d)
    cu = [0] + np.cumsum(rows).tolist()
    q = normal(g, cu[-1], H * G, d).bfloat16()
    # (the row kernel would take more than 16 ranges, large tiles take 16 at most)
    ranges = ts.load_cache().ts_cache_attn_workspace(len(rows), max(rows), max(lens), cu[-1], H, H * G, d, 0) // (cu[-1] * H * G * 4 * (d + 1))
    assert 1 < ranges <= 16
    args = (q, cache, ints(cu), max(rows), ints(table), ints(lens), max(lens))
    o, lse = ts.ts_cache_attn(*args, return_lse=True)
    o2, lse2 = ts.ts_cache_attn(*args, return_lse=True, num_splits=5)
    assert (o.float() - o2.float()).abs().max() <= 4 * 2.0 ** -8 * 6
    assert (lse - lse2).abs().max() <= 1e-4
    assert same(ts.ts_cache_attn(*args, return_lse=True), [o, lse])
