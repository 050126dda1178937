"""The 8-bit session cache on the GPU against its plain 64-bit reference (cache_ref.py): append and evict bit for
bit, attention and the tokens' weights within bounds derived from the roundings; a session's life through all
of them; sessions and pages that break the rules; graphs, streams, validation mode, pools beyond 4 GiB."""
import math

import numpy as np
import pytest
import torch

import cache_ref as R

pytestmark = pytest.mark.gpu

ts = pytest.importorskip("paper_2606_19271_amd")

PAGE = 64


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ts.load_cache()
    return torch.device("cuda:0")


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def offsets(rows):
    return [0] + list(np.cumsum(rows).tolist())


def normal(g, *shape):
    return torch.randn(shape, generator=g)


def make_pool(g, pages, H, d, spread=3):
    """A pool of random values, page exponents uneven by a few powers of two, uneven weights."""
    cache = ts.session_cache(pages, H, d)
    for name in ("k", "v"):
        x = normal(g, pages, H, PAGE, d).numpy() * 2.0
        e = np.array([[R.exponent(x[p, h]) for h in range(H)] for p in range(pages)])
        b = R.round_e4m3(x * 2.0 ** (127 - e)[:, :, None, None])
        shift = torch.randint(-spread, spread + 1, (pages, H), generator=g).numpy()
        getattr(cache, name).view(torch.uint8).copy_(torch.from_numpy(b))
        getattr(cache, name + "_exp").copy_(torch.from_numpy((e + shift).astype(np.uint8)))
    cache.weight.copy_(normal(g, pages, H, PAGE) ** 2)
    return cache


def make_table(g, lens, width, pages):
    """Pages of the sessions, scattered over the pool; entries past a session's last page are wild."""
    order = torch.randperm(pages, generator=g).tolist()
    table = []
    for n in lens:
        need = -(-n // PAGE)
        table.append([order.pop() for _ in range(need)] + [-12345, 1 << 30][:max(0, min(2, width - need))]
                     + [-1] * max(0, width - need - 2))
    return table, order


def bf16(x):
    return x.to(torch.bfloat16)


def check_pool(cache, want):
    for name in ("k", "v"):
        assert R.same_values(getattr(cache, name).view(torch.uint8).cpu().numpy(), getattr(want, name)), name
    for name in ("k_exp", "v_exp", "weight"):
        np.testing.assert_array_equal(getattr(cache, name).cpu().numpy(), getattr(want, name), err_msg=name)


# ---- append

APPENDS = [  # (lens, rows)
    ([0], [1]), ([0], [64]), ([63], [1]), ([64], [1]), ([5], [300]), ([0, 70, 128, 191], [0, 57, 64, 66]),
    ([10, 0, 63, 64, 1], [1, 1, 1, 1, 1]), ([0, 0], [0, 0]), ([500, 3], [0, 129])]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,rows", APPENDS)
@pytest.mark.parametrize("gain", [-6, 0, 5])
def test_append(lens, rows, d, gain):
    g = torch.Generator().manual_seed(len(lens) * 100 + sum(rows) + d + gain)
    H, width = 3, max(-(-(a + b) // PAGE) for a, b in zip(lens, rows)) + 1
    pages = sum(-(-(a + b) // PAGE) for a, b in zip(lens, rows)) + 3
    cache = make_pool(g, pages, H, d)
    table, _ = make_table(g, [a + b for a, b in zip(lens, rows)], width, pages)
    cu = offsets(rows)
    # every token and channel at a magnitude of its own, so that a page's elements meet subnormals of its scale
    k = bf16(normal(g, cu[-1], H, d) * torch.exp2(gain + 2 * normal(g, cu[-1], H, 1)))
    v = bf16(normal(g, cu[-1], H, d) * 2.0 ** gain)
    want = R.Pool.of(cache)
    new = ts.ts_cache_append(cache, k.cuda(), v.cuda(), ints(cu), max(rows), ints(table), ints(lens))
    ref = R.append(want, k.double().numpy(), v.double().numpy(), cu, table, lens, width)
    assert new.tolist() == ref
    check_pool(cache, want)


@pytest.mark.parametrize("d", [64, 128])
def test_append_edges_of_the_format(d):
    """Zeros, the smallest and largest magnitudes, magnitudes around 448 * 2^n, ties, infinities and NaN."""
    H = 2
    edge = torch.zeros(8 * 64, H, d)
    edge[64:128, 0] = 2.0 ** -133           # below the least scale's smallest value
    edge[128:192, 0, 0] = 2.0 ** 126
    edge[192:256, 1, 3] = 448.0
    edge[256, 1, 3] = 449.0 + 1             # bfloat16 450: one more power of two for the page
    edge[320:384, 0] = torch.linspace(0, 20, d)  # ties among them
    edge[384, 0, 1], edge[385, 0, 2], edge[386, 0, 3] = math.inf, -math.inf, math.nan
    edge[384:448, 1] = math.inf             # a page of nothing finite
    edge[448:512] = -0.0
    cache = ts.session_cache(9, H, d)
    want = R.Pool.of(cache)
    x = bf16(edge)
    table = [[8, 0, 7, 1, 6, 2, 5, 3]]
    new = ts.ts_cache_append(cache, x.cuda(), x.flip(1).contiguous().cuda(), ints([0, 512]), 512, ints(table), ints([0]))
    with np.errstate(invalid="ignore"):
        R.append(want, x.double().numpy(), x.flip(1).double().numpy(), [0, 512], table, [0], 8)
    assert new.tolist() == [512]
    check_pool(cache, want)


def test_append_raises_a_page_s_exponent_step_by_step():
    """Single tokens of growing magnitude into one page: older tokens are rounded again at each rise."""
    d, H = 64, 1
    cache = ts.session_cache(1, H, d)
    want = R.Pool.of(cache)
    g = torch.Generator().manual_seed(4)
    lens = [0]
    for j in range(20):
        x = bf16(normal(g, 1, H, d) * 2.0 ** (j if j % 3 else -j))
        dev = ts.ts_cache_append(cache, x.cuda(), x.cuda(), ints([0, 1]), 1, ints([[0]]), ints(lens))
        lens = R.append(want, x.double().numpy(), x.double().numpy(), [0, 1], [[0]], lens, 1)
        assert dev.tolist() == lens
        check_pool(cache, want)


def test_append_without_weights_and_into_out():
    g = torch.Generator().manual_seed(9)
    cache = make_pool(g, 4, 2, 64)
    want = R.Pool.of(cache)
    want.weight = None
    x = bf16(normal(g, 70, 2, 64))
    out = ints([7])
    r = ts.ts_cache_append(cache._replace(weight=None), x.cuda(), x.cuda(), ints([0, 70]), 70, ints([[3, 1]]), ints([2]), out=out)
    R.append(want, x.double().numpy(), x.double().numpy(), [0, 70], [[3, 1]], [2], 2)
    assert r is out and out.tolist() == [72]
    want.weight = cache.weight.cpu().numpy()
    check_pool(cache, want)


def test_append_skips_sessions_and_pages_that_break_the_rules():
    """Lengths and rows out of bounds, sessions that outgrow their table, pages outside the pool."""
    g = torch.Generator().manual_seed(5)
    H, d, width = 2, 64, 2
    rows = [3, 3, 3, 40, 80]
    lens = [-1, 129, 126, 60, 10]  # negative; beyond the table; 126 + 3 outgrows it; good; one page is bad
    cache = make_pool(g, 8, H, d)
    table = [[0, 1], [0, 1], [0, 1], [2, 3], [5, 99]]
    cu = offsets(rows)
    x = bf16(normal(g, cu[-1], H, d))
    want = R.Pool.of(cache)
    new = ts.ts_cache_append(cache, x.cuda(), x.cuda(), ints(cu), 80, ints(table), ints(lens))
    ref = R.append(want, x.double().numpy(), x.double().numpy(), cu, table, lens, width)
    assert new.tolist() == ref == [-1, 129, 126, 100, 90]
    check_pool(cache, want)
    # rows outside the packed tensor, more than the stated most, and running backwards
    before = R.Pool.of(cache)
    new = ts.ts_cache_append(cache, x.cuda(), x.cuda(), ints([-5, 2, 1, 90, 1 << 30]), 80, ints(table[:4]), ints([0, 0, 0, 0]))
    assert new.tolist() == [0, 0, 0, 0]
    check_pool(cache, before)


# ---- attention

def attn_bounds(q, pool, cu, table, lens, scale, size, o, lse):
    """How far o and lse may be off.  A score is a sum of d exact products of 16-bit operands in fp32 and one fused
    multiply-add: off by at most (d + 2) 2^-24 of the sum of its terms' magnitudes (S), which shifts ln of a weight by as
    much; exp2 and the sums add a few 2^-23.  The weights are rounded to bfloat16 (half a step, 2^-8) before they
    meet the values, and the result is rounded once more.  Weights are formed as 2^-39 of the largest one's size
    (room for later, larger ones before the maximum is moved), and those under 2^-126, the least normal
    number, may be lost: n weights of less than 2^-87 each, times the largest value, whose sum the row's total,
    at least 1, divides."""
    d = q.shape[2]
    S, gone = np.zeros(lse.shape), np.zeros(lse.shape)
    G = q.shape[1] // pool.k.shape[1]
    for s, n in enumerate(lens):
        for hq in range(q.shape[1]):
            if n:
                k = np.abs(np.nan_to_num(pool.tokens("k", table[s], n, hq // G))).max(0)
                S[cu[s]:cu[s + 1], hq] = abs(scale) * (np.abs(q[cu[s]:cu[s + 1], hq]) @ k)
                gone[cu[s]:cu[s + 1], hq] = n * 2.0 ** -87 * np.abs(np.nan_to_num(pool.tokens("v", table[s], n, hq // G))).max()
    shift = (d + 2) * 2.0 ** -24 * S + 2.0 ** -20
    return (2.0 ** -8 + 2 * shift)[..., None] * size + 2.0 ** -8 * np.abs(o) + gone[..., None], shift + 2.0 ** -22 * np.abs(np.nan_to_num(lse, neginf=0))


def run_attn(g, rows, lens, H, G, d, scale=None, num_splits=0, max_extra=0):
    width = max(1, max(-(-n // PAGE) for n in lens)) + 1
    pages = sum(-(-n // PAGE) for n in lens) + 2
    cache = make_pool(g, pages, H, d)
    table, _ = make_table(g, lens, width, pages)
    cu = offsets(rows)
    q = bf16(normal(g, cu[-1], H * G, d))
    scale = 1 / math.sqrt(d) if scale is None else scale
    scale = float(np.float32(scale))
    o, lse = ts.ts_cache_attn(q.cuda(), cache, ints(cu), max(rows) + max_extra, ints(table), ints(lens),
                              min(max(lens) + max_extra, width * PAGE), scale=scale, return_lse=True, num_splits=num_splits)
    pool, q64 = R.Pool.of(cache), q.double().numpy()
    ro, rl, size = R.attend(pool, q64, cu, table, lens, scale)
    bo, bl = attn_bounds(q64, pool, cu, table, lens, scale, size, ro, rl)
    assert np.array_equal(np.isneginf(rl), np.isneginf(lse.cpu().numpy()))
    off = np.abs(o.double().cpu().numpy() - ro)
    assert np.all(off <= bo), (off / np.maximum(bo, 1e-300)).max()
    fine = ~np.isneginf(rl)
    off = np.abs(lse.double().cpu().numpy() - rl)[fine]
    assert np.all(off <= bl[fine]), (off / bl[fine]).max()
    return cache, table, cu, q, o, lse


SHAPES = [  # (rows, lens)
    ([1], [1]), ([1], [64]), ([1], [65]), ([3], [2000]), ([16], [63]), ([17], [129]), ([33], [640]), ([65], [100]),
    ([1, 1, 1, 1], [300, 0, 1, 1000]), ([5, 0, 40, 2], [77, 9, 0, 513]), ([256], [256]), ([257], [1025]),
    ([300, 31, 100], [700, 129, 64])]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,G", [(2, 1), (1, 3), (2, 8)])
@pytest.mark.parametrize("rows,lens", SHAPES)
def test_attn(rows, lens, H, G, d):
    g = torch.Generator().manual_seed(sum(rows) + 7 * sum(lens) + H + G + d)
    run_attn(g, rows, lens, H, G, d, max_extra=(sum(lens) % 3) * 40)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scale", [0.0, -0.2, 1.5, 8.0])
@pytest.mark.parametrize("rows,lens", [([2, 1], [130, 400]), ([70], [333]), ([300], [450])])
def test_attn_scales(scale, rows, lens, d):
    run_attn(torch.Generator().manual_seed(int(10 * scale) + 100 + d), rows, lens, 2, 1, d, scale=scale)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 3, 7, 16, 64])
@pytest.mark.parametrize("rows,lens", [([1, 2], [1000, 70]), ([40], [900]), ([260, 3], [1300, 0])])
def test_attn_splits(n, rows, lens, d):
    """Forced page ranges, many of them empty."""
    run_attn(torch.Generator().manual_seed(n + d), rows, lens, 2, 2, d, num_splits=n)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,lens,H,G", [
    ([280], [8000], 1, 1), ([512], [16_000], 1, 1), ([257, 40], [6001, 5999], 2, 1),  # items cut several times
    ([70, 300, 0, 33, 1], [5000, 900, 4000, 17_000, 0], 1, 2), ([35], [20_001], 2, 3),
    ([40, 1] * 40, [300, 700] * 40, 1, 1), ([70, 1] * 40, [300, 700] * 40, 1, 1), ([33], [63], 1, 1), ([65], [63], 1, 1),
    ([600], [0], 1, 1), ([310, 90], [9000, 2000], 1, 1), ([150, 289], [3000, 7000], 2, 2), ([301], [4000], 1, 1),
    # enough work for shares
    ([280, 90], [9000, 2000], 32, 1), ([70, 300, 0, 33, 1], [5000, 900, 4000, 12_000, 0], 14, 2), ([70, 1] * 40, [300, 2600] * 40, 5, 1),
    ([35, 100], [20_001, 100], 16, 3), ([600, 40], [0, 9000], 24, 1), ([257, 320], [6001, 5999], 32, 1)])
def test_attn_divided_work(rows, lens, H, G, d):
    """Many rows whose work the library divides, into ranges of keys or into equal shares, wherever those cut a row tile's
    keys: as the reference has it, and twice the same result."""
    g = torch.Generator().manual_seed(sum(rows) + sum(lens) + d)
    cache, table, cu, q, o, lse = run_attn(g, rows, lens, H, G, d)
    def call(**kw):
        return ts.ts_cache_attn(q.cuda(), cache, ints(cu), max(rows), ints(table), ints(lens), max(max(lens), 1),
                                return_lse=True, **kw)
    for x, y in zip(call(), (o, lse)):
        assert torch.equal(x, y)


def test_attn_takes_a_smaller_workspace(monkeypatch):
    """The library's own choice falls back to whole row tiles, and to fewer ranges, as the caller's memory goes."""
    g = torch.Generator().manual_seed(3)
    lib = ts.load_cache()
    for rows, lens in (([300], [3000]), ([3], [3000]), ([300, 40], [3000, 500])):
        cache, table, cu, q, o, lse = run_attn(g, rows, lens, 1, 1, 128)
        args = (q.cuda(), cache, ints(cu), max(rows), ints(table), ints(lens), max(lens))
        def call(size, **kw):
            with monkeypatch.context() as m:
                m.setattr(lib, "ts_cache_attn_workspace", lambda *a: size)
                return ts.ts_cache_attn(*args, **kw)
        whole = ts.ts_cache_attn(*args, num_splits=1)
        need = lib.ts_cache_attn_workspace(len(rows), max(rows), max(lens), cu[-1], 1, 1, 128, 0)
        assert need > 0 and torch.equal(call(need), o) and torch.equal(call(0), whole)
        # two results, each off by a rounding of the weights and one of the result: 2^-8 of an average of the values' sizes each
        size = max(np.abs(R.Pool.of(cache).tokens("v", table[s], lens[s], 0)).max() for s in range(len(rows)))
        assert (call(need - 1).float() - whole.float()).abs().max() <= 2 * 2 * 2.0 ** -8 * size
        with pytest.raises(RuntimeError):
            call(0, num_splits=2)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [3, 300])
def test_attn_rising_scores(d, rows):
    """Keys that grow along the session, so that the running maximum moves in every page, by far at the end."""
    g = torch.Generator().manual_seed(d + rows)
    H, n = 1, 700
    cache = ts.session_cache(12, H, d)
    grow = torch.linspace(0.1, 6, n)[:, None, None]
    grow[-30:] *= 4
    k, v = bf16(normal(g, 1, H, d) * grow + 0.1 * normal(g, n, H, d)), bf16(normal(g, n, H, d))
    table = [list(range(11))]
    ts.ts_cache_append(cache, k.cuda(), v.cuda(), ints([0, n]), n, ints(table), ints([0]))
    q = bf16(k[-1:].float().repeat(rows, 1, 1) * (0.2 + torch.rand(rows, 1, 1, generator=g)))
    scale = float(np.float32(0.3))
    o, lse = ts.ts_cache_attn(q.cuda(), cache, ints([0, rows]), rows, ints(table), ints([n]), n, scale=scale, return_lse=True)
    pool, q64 = R.Pool.of(cache), q.double().numpy()
    ro, rl, size = R.attend(pool, q64, [0, rows], table, [n], scale)
    bo, bl = attn_bounds(q64, pool, [0, rows], table, [n], scale, size, ro, rl)
    assert np.all(np.abs(o.double().cpu().numpy() - ro) <= bo)
    assert np.all(np.abs(lse.double().cpu().numpy() - rl) <= bl)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [2, 290])
def test_attn_ignores_what_lies_past_a_session(d, rows):
    """NaN bytes in the slots past the end, wild page numbers past the last page, and pages of other
    sessions that are NaN (page 0 among them) change nothing."""
    g = torch.Generator().manual_seed(d + rows)
    lens = [97, 64, 500]
    width, pages, H = 9, 14, 2
    cache = make_pool(g, pages, H, d)
    table, free = make_table(g, lens, width, pages)
    if 0 not in free:  # page 0 is nobody's
        for row in table:
            row[:] = [free[0] if p == 0 else p for p in row]
        free[0] = 0
    cu = offsets([rows] * 3)
    q = bf16(normal(g, cu[-1], H, d)).cuda()
    args = (q, cache, ints(cu), rows, ints(table), ints(lens), 512)
    a = ts.ts_cache_attn(*args, return_lse=True)
    for s, n in enumerate(lens):
        if n % PAGE:
            for x in (cache.k, cache.v):
                x.view(torch.uint8)[table[s][n // PAGE], :, n % PAGE:] = 0x7f
    for p in free:
        cache.k_exp[p], cache.v_exp[p] = 255, 255
    b = ts.ts_cache_attn(*args, return_lse=True)
    assert torch.equal(a[0].view(torch.int16), b[0].view(torch.int16)) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,splits", [(2, 0), (2, 5), (300, 0), (300, 1), (300, 3)])
def test_attn_bad_sessions_and_pages(d, rows, splits):
    """Sessions that break the rules leave their rows; pages outside the pool, and pages of exponent 255, make
    theirs NaN; the others are as without them."""
    g = torch.Generator().manual_seed(d + rows + splits)
    H, G, pages, width = 2, 1, 12, 4
    cache = make_pool(g, pages, H, d)
    table = [[0, 1, 2, 3], [4, 5, 6, 7], [8, 99, 9, -1], [10, 11, -7, 0], [4, 5, 6, 7], [1, 2, 3, 9], [4, 5, 6, 7]]
    lens = [200, -3, 190, 130, 257, 100, 250]
    cache.v_exp[2, 1] = 255
    cu = offsets([rows] * 7)
    q = bf16(normal(g, cu[-1], H * G, d)).cuda()
    out = torch.full_like(q, 7.0)
    lse = torch.full((cu[-1], H), 7.0, device="cuda")
    ts.ts_cache_attn(q, cache, ints(cu), rows, ints(table), ints(lens), 256, out=out, lse=lse, num_splits=splits)
    pool = R.Pool.of(cache)
    ok = [0, 5, 6]
    ro, rl, size = R.attend(pool, q.double().cpu().numpy(), cu, [t if i in ok else [0] * 4 for i, t in enumerate(table)],
                            [n if i in ok else 0 for i, n in enumerate(lens)], 1 / math.sqrt(d))
    o, ls = out.double().cpu().numpy(), lse.cpu().numpy()
    for s in range(7):
        r = slice(cu[s], cu[s + 1])
        if s in (1, 4):
            assert np.all(o[r] == 7) and np.all(ls[r] == 7), s
        elif s in (2, 3):
            assert np.all(np.isnan(o[r])) and np.all(np.isnan(ls[r])), s
        else:
            nan = np.isnan(ro[r])
            assert np.array_equal(nan, np.isnan(o[r])) and nan.any() == (s in (0, 5))
            np.testing.assert_allclose(np.where(nan, 0, o[r]), np.where(nan, 0, ro[r]), atol=0.05 * np.nanmax(np.abs(ro[r])), rtol=0)
            np.testing.assert_allclose(ls[r], rl[r], atol=1e-3, rtol=0)
    # rows outside the packed tensor, more than the stated most, backwards: nothing is written
    out.fill_(7.0)
    bad = ints([-1, rows, rows - 1, 1 << 30])
    ts.ts_cache_attn(q, cache, bad, rows, ints(table[:3]), ints([64, 64, 64]), 256, out=out, num_splits=splits)
    assert torch.all(out == 7.0)


# ---- the tokens' weights

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,G", [(2, 1), (1, 5)])
@pytest.mark.parametrize("rows,lens", [([1], [1]), ([1, 1, 3], [64, 200, 65]), ([40, 0, 7], [130, 77, 0]), ([20, 31, 17], [300, 129, 64]), ([257], [700]),
                                       ([1000], [100])])
@pytest.mark.parametrize("scale", [None, -0.3])
def test_weigh(rows, lens, H, G, d, scale):
    g = torch.Generator().manual_seed(sum(rows) + sum(lens) + d)
    cache, table, cu, q, _, lse = run_attn(g, rows, lens, H, G, d, scale=scale)
    pool = R.Pool.of(cache)
    scale = float(np.float32(1 / math.sqrt(d) if scale is None else scale))
    want = R.weigh(pool, q.double().numpy(), lse.double().cpu().numpy(), cu, table, lens, scale)
    out = torch.full_like(cache.weight, 5.0)
    args = (q.cuda(), lse, cache, ints(cu), max(rows), ints(table), ints(lens), max(lens))
    got = ts.ts_cache_weigh(*args, scale=scale, out=out)
    assert got is out
    got = got.double().cpu().numpy()
    live = np.zeros(want.shape, bool)
    for s, n in enumerate(lens):
        for j in range(n):
            live[table[s][j // PAGE], :, j % PAGE] = True
    assert np.all(got[~live] == 5)
    # scores as in attn_bounds; sums of up to `rows * G` terms and the weight before in fp32: 2^-24 each of the result
    most = max(abs(scale) * float((q.float().abs().sum(2).max())) * 64, 1.0)
    rel = (d + 2) * 2.0 ** -24 * most + (max(rows) * G + 8) * 2.0 ** -24 + 2.0 ** -20
    off = np.abs(got - want)[live] / np.maximum(np.abs(want[live]), 1e-30)
    assert off.size == 0 or off.max() <= rel, (off.max(), rel)
    # in place, and each query row hands out a weight of one
    before = cache.weight.double().cpu().numpy()[live].sum()
    assert ts.ts_cache_weigh(*args, scale=scale) is cache.weight
    after = cache.weight.double().cpu().numpy()
    np.testing.assert_array_equal(after[live], got[live])
    given = sum(a * H * G for a, b in zip(rows, lens) if b)
    assert abs(after[live].sum() - before - given) <= 1e-4 * max(given, before, 1)


@pytest.mark.parametrize("d,G,rows,lens", [(128, 1, [70, 1, 0], [60_000, 30_001, 5_000]), (64, 3, [200, 3, 64], [50_000, 999, 60_064]),
                                           (128, 5, [13, 300], [64_000, 20_000])])
def test_weigh_many_keys(d, G, rows, lens):
    """Enough keys for several groups of pages to a workgroup, sessions of unequal length, a bad page among them."""
    g = torch.Generator().manual_seed(d + G)
    H = 2
    width = -(-max(lens) // PAGE)
    pages = sum(-(-n // PAGE) for n in lens) + 2
    cache = make_pool(g, pages, H, d)
    table, _ = make_table(g, lens, width, pages)
    table[0][100] = pages + 7
    cu = offsets(rows)
    q = bf16(normal(g, cu[-1], H * G, d))
    lse = (10 + normal(g, cu[-1], H * G)).cuda()
    pool = R.Pool.of(cache)
    scale = float(np.float32(1 / math.sqrt(d)))
    with np.errstate(invalid="ignore"):
        want = R.weigh(pool, q.double().numpy(), lse.double().cpu().numpy(), cu, table, lens, scale)
    out = torch.full_like(cache.weight, 5.0)
    ts.ts_cache_weigh(q.cuda(), lse, cache, ints(cu), max(rows), ints(table), ints(lens), max(lens), out=out)
    got = out.double().cpu().numpy()
    live = np.zeros(want.shape, bool)
    for s, n in enumerate(lens):
        for j in range(0, n, PAGE):
            if table[s][j // PAGE] < pages:
                live[table[s][j // PAGE], :, :min(PAGE, n - j)] = True
    assert np.all(got[~live] == 5)
    most = abs(scale) * float((q.float().abs().sum(2).max())) * 64
    rel = (d + 2) * 2.0 ** -24 * most + (max(rows) * G + 8) * 2.0 ** -24 + 2.0 ** -20
    # (an lse that is not these rows' own lets single weights pass the largest float32: those are infinite)
    over = live & (want > np.finfo(np.float32).max)
    assert np.all(np.isinf(got[over]))
    live &= ~over
    assert (np.abs(got - want)[live] / want[live]).max() <= rel


@pytest.mark.parametrize("rows", [1, 30, 64])
def test_weigh_long_sessions_of_many_heads(rows):
    """So many heads that a workgroup has all of a session's pages, and each wave more than 64 of them, in a pool beyond
    2 GiB: against the kernel for many rows, whose choice goes by the stated most of them."""
    H, d, n = 2048, 64, 16_500
    pages = -(-n // PAGE) + 1
    g = torch.Generator(device="cuda").manual_seed(rows)
    cache = ts.session_cache(pages, H, d)
    cache.k.view(torch.uint8).random_(0, 100, generator=g)
    cache.k_exp.fill_(122)
    cache.weight.random_(0, 5, generator=g)
    table = torch.randperm(pages, generator=g, device="cuda").int()[None].contiguous()
    q = torch.randn(rows, H, d, generator=g, device="cuda").bfloat16()
    lse = torch.full((rows, H), 6.0, device="cuda")
    a, b = cache.weight.clone(), cache.weight.clone()
    for out, most in ((a, rows), (b, 65)):
        ts.ts_cache_weigh(q, lse, cache, ints([0, rows]), most, table, ints([n]), n, out=out)
    assert not torch.equal(a, cache.weight)
    # scores good to (d + 2) 2^-24 of their terms' sum (below 2^9 here), which shifts a weight by as much relatively
    torch.testing.assert_close(a, b, rtol=2 * 66 * 2.0 ** -15, atol=0)


@pytest.mark.parametrize("rows", [2, 20, 100])
@pytest.mark.parametrize("d", [64, 128])
def test_weigh_of_nothing_finite(d, rows):
    """A session without rows keeps its weights, NaN keys or not; infinite queries and an infinite lse as the formula has
    them, next to sessions that they do not touch."""
    g = torch.Generator().manual_seed(d + rows)
    H = 2
    cache = make_pool(g, 12, H, d)
    cache.k_exp[1] = 255
    table, lens, cu = ints([[0, 1, 2], [3, 4, 5], [6, 7, 8], [9, 10, 11]]), [190, 150, 192, 65], [0, 0, rows, rows + 1, rows + 2]
    q = bf16(normal(g, rows + 2, H, d))
    q[rows, 0, 0] = math.inf
    lse = torch.full((rows + 2, H), 3.0)
    lse[rows + 1, 0], lse[rows + 1, 1] = math.inf, -math.inf
    want, before = R.Pool.of(cache), cache.weight.clone()
    ts.ts_cache_weigh(q.cuda(), lse.cuda(), cache, ints(cu), max(rows, 1), table, ints(lens), 192)
    after = cache.weight
    assert torch.equal(after[:3], before[:3])
    k = [want.tokens("k", [6, 7, 8], 192, h) for h in range(H)]
    sign = np.sign(k[0][:, 0])
    got = after[6:9, 0].reshape(-1).cpu().numpy()
    assert np.all(np.isposinf(got[sign > 0])) and np.all(np.isnan(got[sign == 0]))
    assert np.array_equal(got[sign < 0], before[6:9, 0].reshape(-1).cpu().numpy()[sign < 0])
    assert torch.equal(after[9, 0], before[9, 0]) and torch.all(torch.isposinf(after[9, 1]))
    assert torch.equal(after[10:], before[10:]) is False and torch.equal(after[10, :, 1:], before[10, :, 1:])
    assert torch.all(torch.isfinite(after[3:5])) and torch.all(torch.isfinite(after[6:9, 1]))


def test_weigh_bad_sessions_and_pages():
    g = torch.Generator().manual_seed(3)
    H, d = 2, 64
    cache = make_pool(g, 8, H, d)
    table = [[0, 1], [2, 77], [4, 5], [6, 7]]
    lens = [100, 128, 129, 5]
    cu = [0, 3, 6, 9, 50]
    q = bf16(normal(g, 9, H, d)).cuda()
    lse = torch.full((9, H), 9.0, device="cuda")
    before = cache.weight.cpu().numpy()
    ts.ts_cache_weigh(q, lse, cache, ints(cu), 3, ints(table), ints(lens), 128)
    after = cache.weight.cpu().numpy()
    changed = (after != before).any(axis=(1, 2))
    assert changed.tolist() == [True, True, True, False, False, False, False, False]


# ---- eviction

EVICTIONS = [  # (lens, keep, first, last)
    ([1], 1, 0, 0), ([100], 64, 0, 0), ([65], 64, 0, 0), ([300, 20, 0, 129], 129, 5, 30), ([1000], 130, 130, 0),
    ([1000], 70, 0, 70), ([700, 701], 699, 1, 1), ([3000, 64], 1, 0, 0), ([200], 0, 0, 0), ([640], 500, 64, 64)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,keep,first,last", EVICTIONS)
@pytest.mark.parametrize("ties", [False, True])
def test_evict(lens, keep, first, last, ties, d):
    g = torch.Generator().manual_seed(sum(lens) + keep + d)
    H, width, new_width = 2, max(-(-n // PAGE) for n in lens) + 1, -(-keep // PAGE) + 1
    pages = sum(-(-n // PAGE) for n in lens) + new_width * len(lens) + 1
    cache = make_pool(g, pages, H, d, spread=9)
    if ties:
        cache.weight.copy_((cache.weight * 2).round() / 2)
    table, free = make_table(g, lens, width, pages)
    new_table = [[free.pop() for _ in range(new_width - 1)] + [-9] for _ in lens]
    want = R.Pool.of(cache)
    new, kept = ts.ts_cache_evict(cache, ints(table), ints(lens), max(lens), ints(new_table), keep, first, last)
    ref, ref_kept = R.evict(want, table, lens, new_table, keep, first, last)
    assert new.tolist() == ref
    np.testing.assert_array_equal(kept.cpu().numpy(), ref_kept)
    check_pool(cache, want)


def test_evict_orders_every_kind_of_weight():
    """Infinities, NaN, both zeros, negatives, subnormals, and the largest finite weights; all equal weights."""
    d, H, n = 64, 3, 320
    g = torch.Generator().manual_seed(8)
    cache = make_pool(g, 12, H, d)
    special = torch.tensor([math.inf, -math.inf, math.nan, 0.0, -0.0, -1.0, 1e-42, -1e-42, 3.4e38, -3.4e38])
    pick = torch.randint(0, 10, (12, PAGE), generator=g)
    cache.weight[:, 0] = special[pick].cuda()
    cache.weight[:, 1] = 0.0
    for keep in (7, 100, 319):
        table, new_table = [[3, 1, 4, 0, 5]], [[6, 7, 8, 9, 10]]
        want = R.Pool.of(cache)
        new, kept = ts.ts_cache_evict(cache, ints(table), ints([n]), n, ints(new_table), keep, 2, 3)
        ref, ref_kept = R.evict(want, table, [n], new_table, keep, 2, 3)
        assert new.tolist() == ref
        np.testing.assert_array_equal(kept.cpu().numpy(), ref_kept)
        check_pool(cache, want)


def test_evict_long_session():
    """Longer than the selecting workgroup's registers or LDS could hold, with many equal weights."""
    n, H, d, keep = 70001, 1, 64, 33333
    pages = -(-n // PAGE)
    cache = ts.session_cache(pages + -(-keep // PAGE), H, d)
    g = torch.Generator(device="cuda").manual_seed(1)
    cache.weight.copy_((torch.rand(cache.weight.shape, generator=g, device="cuda") * 500).round())
    table, new_table = ints([list(range(pages))]), ints([list(range(pages, pages + -(-keep // PAGE)))])
    new, kept = ts.ts_cache_evict(cache, table, ints([n]), n, new_table, keep, 100, 200)
    w = cache.weight[:pages, 0].reshape(-1)[:n].clone()
    w[:100] = w[n - 200:] = math.inf
    want = torch.sort(w, descending=True, stable=True).indices[:keep].sort().values
    assert new.tolist() == [keep] and torch.equal(kept[0, 0].long(), want)


def test_evict_bad_sessions_and_pages():
    g = torch.Generator().manual_seed(2)
    H, d, keep = 2, 64, 70
    cache = make_pool(g, 12, H, d)
    table = [[0, 1, 2], [0, 1, 2], [3, 500, 4], [0, 1, 2]]
    lens = [193, -1, 150, 140]
    new_table = [[5, 6], [5, 6], [7, 8], [9, -1]]
    want = R.Pool.of(cache)
    new, kept = ts.ts_cache_evict(cache, ints(table), ints(lens), 192, ints(new_table), keep, 4, 4)
    assert new.tolist() == [193, -1, 70, 70]
    assert torch.all(kept[:2] == -1)
    with np.errstate(invalid="ignore"):
        _, ref = R.evict(want, table[2:], lens[2:], new_table[2:], keep, 4, 4)
    np.testing.assert_array_equal(kept[2:].cpu().numpy(), ref)
    check_pool(cache, want)


# ---- together

@pytest.mark.parametrize("d,G", [(64, 1), (128, 2)])
def test_a_session_s_life(d, G):
    """Chunks appended, attended, weighed, and the sessions cut down whenever they pass a budget: every step
    against the reference, which follows the device's own lse and weights."""
    g = torch.Generator().manual_seed(d)
    H, width, budget, keep, pages = 2, 8, 330, 200, 64
    cache = ts.session_cache(pages, H, d)
    free = list(range(pages))
    lens, table = [0, 0, 0], [[] for _ in range(3)]
    scale = float(np.float32(1 / math.sqrt(d)))
    for step in range(5):
        rows = [[60, 130, 1], [90, 1, 64], [128, 100, 0], [33, 150, 129], [64, 64, 64]][step]
        for s in range(3):
            while len(table[s]) * PAGE < lens[s] + rows[s]:
                table[s].append(free.pop(0))
        full = [t + [-1] * (width - len(t)) for t in table]
        cu = offsets(rows)
        k, v = bf16(normal(g, cu[-1], H, d)), bf16(normal(g, cu[-1], H, d))
        q = bf16(normal(g, cu[-1], H * G, d))
        want = R.Pool.of(cache)
        dev_lens = ts.ts_cache_append(cache, k.cuda(), v.cuda(), ints(cu), max(rows), ints(full), ints(lens))
        lens = R.append(want, k.double().numpy(), v.double().numpy(), cu, full, lens, width)
        assert dev_lens.tolist() == lens
        check_pool(cache, want)
        o, lse = ts.ts_cache_attn(q.cuda(), cache, ints(cu), max(rows), ints(full), dev_lens, width * PAGE, return_lse=True)
        ro, rl, size = R.attend(want, q.double().numpy(), cu, full, lens, scale)
        bo, bl = attn_bounds(q.double().numpy(), want, cu, full, lens, scale, size, ro, rl)
        assert np.all(np.abs(o.double().cpu().numpy() - ro) <= bo)
        assert np.all(np.abs(lse.double().cpu().numpy() - rl) <= bl)
        after = R.weigh(want, q.double().numpy(), lse.double().cpu().numpy(), cu, full, lens, scale)
        ts.ts_cache_weigh(q.cuda(), lse, cache, ints(cu), max(rows), ints(full), dev_lens, width * PAGE)
        np.testing.assert_allclose(cache.weight.cpu().numpy(), after, rtol=1e-4, atol=1e-6)
        if max(lens) > budget:
            want = R.Pool.of(cache)
            new_table = [[free.pop(0) for _ in range(-(-keep // PAGE))] for _ in range(3)]
            dev_lens, kept = ts.ts_cache_evict(cache, ints(full), dev_lens, width * PAGE, ints(new_table), keep, 16, 64)
            lens, ref = R.evict(want, full, lens, new_table, keep, 16, 64)
            assert dev_lens.tolist() == lens
            np.testing.assert_array_equal(kept.cpu().numpy(), ref)
            check_pool(cache, want)
            for s in range(3):
                free += table[s]
                used = -(-lens[s] // PAGE)
                table[s] = new_table[s][:used]
                free += new_table[s][used:]


def test_the_cached_attention_is_the_chunk_call_s_on_the_same_values():
    """The pages' values as packed bfloat16 tensors, through ts_attn_fwd_kvcache: the same attention."""
    g = torch.Generator().manual_seed(6)
    H, d, rows, lens = 4, 128, [100, 300], [513, 900]
    cache, table, cu, q, o, lse = run_attn(g, rows, lens, H, 1, d)
    pool = R.Pool.of(cache)
    k, v = (torch.cat([torch.stack([torch.from_numpy(pool.tokens(n, table[s], lens[s], h)) for h in range(H)], 1)
                       for s in range(2)]).bfloat16().cuda() for n in ("k", "v"))
    o2, lse2 = ts.ts_attn_fwd_kvcache(q.cuda(), k, v, ints(cu), ints(offsets(lens)), max(rows), max(lens), return_lse=True)
    scale = float(o2.float().abs().max())
    assert float((o.float() - o2.float()).abs().max()) <= 3 * 2.0 ** -8 * scale
    assert float((lse - lse2).abs().max()) <= 2.0 ** -8


def test_pages_move_with_the_state_copy():
    """A session's pages suspended to pinned memory and resumed at other page numbers: the same attention."""
    g = torch.Generator().manual_seed(7)
    H, d, lens = 2, 64, [300]
    cache, table, cu, q, o, _ = run_attn(g, [5], lens, H, 1, d)
    fresh = ts.session_cache(20, H, d)
    page_bytes = H * PAGE * d
    where = [11, 3, 19, 7, 0]
    for a, b in ((cache.k, fresh.k), (cache.v, fresh.v)):
        host = torch.empty(5 * page_bytes, dtype=torch.uint8, pin_memory=True)
        ts.ts_state_copy(a, host, [(table[0][i] * page_bytes, i * page_bytes, page_bytes) for i in range(5)])
        ts.ts_state_copy(host, b, [(i * page_bytes, where[i] * page_bytes, page_bytes) for i in range(5)])
    idx = torch.tensor(table[0][:5], device="cuda")
    fresh.k_exp[torch.tensor(where, device="cuda")] = cache.k_exp[idx]
    fresh.v_exp[torch.tensor(where, device="cuda")] = cache.v_exp[idx]
    again = ts.ts_cache_attn(q.cuda(), fresh, ints(cu), 5, ints([where]), ints(lens), 300)
    assert torch.equal(again.view(torch.int16), o.view(torch.int16))


# ---- how the calls run

def chunk_step(g, d=128, H=2, rows=(40, 3), lens=(500, 131)):
    """Tensors of a chunk step: pages, tables, new tokens, queries."""
    width = 12
    cache = make_pool(g, 40, H, d)
    total = [a + b for a, b in zip(rows, lens)]
    table, free = make_table(g, total, width, 40)
    cu = offsets(rows)
    t = {"cache": cache, "cu": ints(cu), "table": ints(table), "lens": ints(list(lens)),
         "new_table": ints([[free.pop() for _ in range(3)] for _ in rows])}
    for n in ("q", "k", "v"):
        t[n] = bf16(normal(g, cu[-1], H, d)).cuda()
    return t


def run_step(t, rows=40, splits=0):
    lens = ts.ts_cache_append(t["cache"], t["k"], t["v"], t["cu"], rows, t["table"], t["lens"])
    o, lse = ts.ts_cache_attn(t["q"], t["cache"], t["cu"], rows, t["table"], lens, 768, return_lse=True, num_splits=splits)
    ts.ts_cache_weigh(t["q"], lse, t["cache"], t["cu"], rows, t["table"], lens, 768)
    new, kept = ts.ts_cache_evict(t["cache"], t["table"], lens, 768, t["new_table"], 150, 10, 20)
    return [lens, o, lse, new, kept]


def clone(t):
    return {k: ts.SessionCache(*(x.clone() for x in v)) if k == "cache" else v.clone() for k, v in t.items()}


def same(a, b):
    def bits(x):
        return x.contiguous().view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32 if x.dtype == torch.float32
                                   else torch.uint8 if x.dtype == torch.float8_e4m3fn else x.dtype)
    return all(torch.equal(bits(x), bits(y)) for x, y in zip(a, b))


@pytest.mark.parametrize("rows", [40, 70])
@pytest.mark.parametrize("splits", [0, 4])
def test_graph_replays(splits, rows):
    """A whole chunk step in one HIP graph, replayed with new inputs and eager work in between: every replay as
    the eager calls."""
    g = torch.Generator().manual_seed(11)
    t = chunk_step(g, rows=(rows, 3))
    run_step(clone(t), rows, splits)  # the device's first call is outside capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run_step(t, rows, splits)
    for i in range(4):
        for n in ("q", "k", "v"):
            t[n].copy_(bf16(normal(g, *t[n].shape)))
        want_t = clone(t)
        want = run_step(want_t, rows, splits)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert same(got, want), i
        assert same(t["cache"], want_t["cache"]), i


@pytest.mark.parametrize("rows,splits", [(40, 6), (70, 0)])
def test_two_streams_at_once(rows, splits):
    """Interleaved steps on two streams share nothing, workspaces included."""
    g = torch.Generator().manual_seed(12)
    ts_ = [chunk_step(g, rows=(rows, 3)), chunk_step(g, rows=(rows, rows), lens=(600, 300))]
    want = [run_step(clone(t), rows, splits) for t in ts_]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ts_]
    got = [None, None]
    work = [[clone(t) for t in ts_] for _ in range(6)]
    torch.cuda.synchronize()
    rounds = []
    for r in range(6):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i] = run_step(work[r][i], rows, splits)
        rounds.append(list(got))
    torch.cuda.synchronize()
    for got in rounds:
        for i in range(2):
            assert same(got[i], want[i])


def test_calls_are_reproducible():
    g = torch.Generator().manual_seed(13)
    t = chunk_step(g)
    a, b = clone(t), clone(t)
    assert same(run_step(a), run_step(b)) and same(a["cache"], b["cache"])


def test_sessions_do_not_depend_on_each_other():
    """A session alone and in a batch (with the same number of page ranges): the same rows, bit for bit."""
    g = torch.Generator().manual_seed(14)
    H, d, lens, rows = 2, 128, [300, 1000, 64], [20, 1, 9]
    cache, table, cu, q, o, lse = run_attn(g, rows, lens, H, 1, d, num_splits=3)
    for s in range(3):
        a, b = ts.ts_cache_attn(q[cu[s]:cu[s + 1]].contiguous().cuda(), cache, ints([0, rows[s]]), 20, ints([table[s]]), ints([lens[s]]),
                                1000, return_lse=True, num_splits=3)
        assert torch.equal(a, o[cu[s]:cu[s + 1]]) and torch.equal(b, lse[cu[s]:cu[s + 1]])


def test_more_sessions_than_lanes():
    g = torch.Generator().manual_seed(15)
    rows = [1 + (i * 7) % 5 for i in range(150)]
    lens = [(i * 37) % 200 for i in range(150)]
    run_attn(g, rows, lens, 1, 1, 64)


def test_more_sessions_than_lanes_in_large_tiles():
    g = torch.Generator().manual_seed(19)
    rows = [(i * 53) % 301 for i in range(70)]
    lens = [(i * 37) % 200 for i in range(70)]
    run_attn(g, rows, lens, 1, 1, 64)


@pytest.mark.parametrize("d,rows,splits", [(64, 40, 1), (128, 40, 1), (64, 70, 1), (128, 70, 1), (128, 70, 0), (128, 290, 2),
                                           (64, 3, 1), (128, 20, 2)])
def test_attn_long_sessions(d, rows, splits):
    """More pages than an item keeps at hand at once; the longer session ends inside a page and inside a tile, and a
    page far behind is outside the pool."""
    g = torch.Generator().manual_seed(d + rows)
    lens = [100_031, 40_000]
    cache, table, cu, q, o, lse = run_attn(g, [rows, 33], lens, 1, 1, d, num_splits=splits)
    table[1][600] = 1 << 29
    o2 = ts.ts_cache_attn(q.cuda(), cache, ints(cu), max(rows, 33), ints(table), ints(lens), max(lens), num_splits=splits)
    assert torch.equal(o2[:rows], o[:rows]) and torch.isnan(o2[rows:]).all()


def test_validation_mode(monkeypatch):
    from paper_2606_19271_amd import _lib
    g = torch.Generator().manual_seed(16)
    t = chunk_step(g)
    monkeypatch.setenv("TS_ATTN_VALIDATE", "1")
    run_step(t)
    lens = t["lens"]
    for bad in ({"lens": ints([-1, 5])}, {"lens": ints([769, 5])}, {"table": torch.full_like(t["table"], 40)}, {"cu": ints([0, 44, 43])},
                {"cu": ints([-1, 40, 43])}, {"cu": ints([0, 40, 44])}):
        u = dict(t, **bad)
        with pytest.raises(ts.TsAttnError) as e:
            ts.ts_cache_attn(u["q"], u["cache"], u["cu"], 40, u["table"], u["lens"], 768)
        assert e.value.status == _lib.TS_ERR_SEGMENTS
        with pytest.raises(ts.TsAttnError):
            ts.ts_cache_append(u["cache"], u["k"], u["v"], u["cu"], 40, u["table"], u["lens"])
    with pytest.raises(ts.TsAttnError):
        ts.ts_cache_evict(t["cache"], t["table"], lens, 768, torch.full_like(t["new_table"], -1), 150)
    with pytest.raises(ts.TsAttnError):  # outgrows its table
        ts.ts_cache_append(t["cache"], t["k"], t["v"], t["cu"], 40, t["table"][:, :8].contiguous(), lens)


def test_pool_beyond_four_gib():
    """Pages whose bytes lie past 2^32 in the pool (and weights past 2^31 elements' bytes)."""
    H, d = 8, 128
    pages = (1 << 32) // (H * PAGE * d) + 64
    cache = ts.session_cache(pages, H, d)
    table = [[pages - 1, pages - 7, 3, pages - 20], [pages - 2, 0, pages - 30, pages - 31]]
    g = torch.Generator().manual_seed(17)
    rows = [200, 130]
    cu = offsets(rows)
    k, v, q = (bf16(normal(g, 330, H, d)) for _ in range(3))
    lens = ts.ts_cache_append(cache, k.cuda(), v.cuda(), ints(cu), 200, ints(table), ints([0, 0]))
    assert lens.tolist() == rows
    idx = torch.tensor(table, device="cuda").reshape(-1)
    small = ts.SessionCache(cache.k.view(torch.uint8)[idx].contiguous().view(torch.float8_e4m3fn),
                            cache.v.view(torch.uint8)[idx].contiguous().view(torch.float8_e4m3fn), cache.k_exp[idx].contiguous(), cache.v_exp[idx].contiguous(),
                            cache.weight[idx].contiguous())
    near = [[0, 1, 2, 3], [4, 5, 6, 7]]
    fresh = ts.session_cache(8, H, d)
    ts.ts_cache_append(fresh, k.cuda(), v.cuda(), ints(cu), 200, ints(near), ints([0, 0]))
    assert same([fresh.k[:3], fresh.k_exp[:3]], [small.k[:3], small.k_exp[:3]])
    for n in (1, 3):
        a = ts.ts_cache_attn(q.cuda(), cache, ints(cu), 200, ints(table), lens, 256, return_lse=True, num_splits=n)
        b = ts.ts_cache_attn(q.cuda(), small, ints(cu), 200, ints(near), lens, 256, return_lse=True, num_splits=n)
        assert same(a, b)
    ts.ts_cache_weigh(q.cuda(), a[1], cache, ints(cu), 200, ints(table), lens, 256)
    ts.ts_cache_weigh(q.cuda(), a[1], small, ints(cu), 200, ints(near), lens, 256)
    assert torch.equal(cache.weight[idx], small.weight)
    new_table = ints([[pages - 40, pages - 41], [1, pages - 42]])
    _, kept = ts.ts_cache_evict(cache, ints(table), lens, 256, new_table, 100, 1, 1)
    big = ts.session_cache(16, H, d)
    for x, y in zip(big, small):
        x.view(torch.uint8 if x.dtype == torch.float8_e4m3fn else x.dtype)[:8] = y.view(torch.uint8 if y.dtype == torch.float8_e4m3fn else y.dtype)
    _, kept2 = ts.ts_cache_evict(big, ints(near), lens, 256, ints([[8, 9], [10, 11]]), 100, 1, 1)
    assert torch.equal(kept, kept2)
    assert torch.equal(cache.k.view(torch.uint8)[pages - 41, :, :36], big.k.view(torch.uint8)[9, :, :36])


def test_another_device_current():
    """The calls run on the pool's device whatever device is current."""
    if torch.cuda.device_count() < 2:
        pytest.skip("one GPU")
    t = chunk_step(torch.Generator().manual_seed(18))
    u = clone(t)
    want = run_step(t)
    with torch.cuda.device(1):
        got = run_step(u)
    assert same(got, want)
