"""The transformer block's calls where they can go wrong: memory that is shared, strided or far apart, values at the ends of bfloat16,
offsets that break the rules, graphs, streams, and a training and a serving step of the calls together."""
import math

import numpy as np
import pytest
import torch

import block_ref as R
from test_gpu_block import ATTN, AXES, attn_inputs, check_attn, near, normal, rng, rope_inputs, same_bits, say

pytestmark = pytest.mark.gpu

ts = pytest.importorskip("paper_2606_19271_amd")


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ts.load()
    ts.load_block()


# ---- norm and rotation


def rope_tol(x, w, angle, interleaved, eps):
    ref, mag = (f(x.double(), None if w is None else w.double(), angle, interleaved, eps) for f in (R.rope, R.rope_slack))
    return ref, R.HALF * ref.abs() + 1.01 * R.FINE * mag


@pytest.mark.parametrize("d", [64, 128])
def test_rope_in_place_within_fused_rows(d):
    say("in place", d)
    T, Hq, Hk = 333, 6, 3
    g = rng(1)
    rows = (normal(g, T, Hq + 2 * Hk + 1, d)).bfloat16()  # (a head's room at the end belongs to nobody)
    was = rows.clone()
    wq, wk = 1 + 0.3 * normal(g, d), 1 + 0.3 * normal(g, d)
    r, pos = ts.rope(AXES[d]), torch.randint(0, 99, (T, 3), generator=g, device="cuda").int()
    q, k = rows[:, :Hq], rows[:, Hq:Hq + Hk]
    new = ts.ts_qk_rope(q, k, pos, r, wq, wk)
    a, b = ts.ts_qk_rope(q, k, pos, r, wq, wk, q_out=q, k_out=k)
    assert a is q and b is k and same_bits(q, new[0]) and same_bits(k, new[1])
    assert same_bits(rows[:, Hq + Hk:], was[:, Hq + Hk:])
    # gradients into another fused tensor, and over their own results' gradients
    dq, dk = normal(g, T, Hq, d).bfloat16(), normal(g, T, Hk, d).bfloat16()
    x, y = was[:, :Hq], was[:, Hq:Hq + Hk]
    new = ts.ts_qk_rope_bwd(dq, dk, x, y, pos, r, wq, wk)
    grads = torch.zeros_like(rows)
    got = ts.ts_qk_rope_bwd(dq, dk, x, y, pos, r, wq, wk, dq=grads[:, :Hq], dk=grads[:, Hq:Hq + Hk])
    assert all(same_bits(u, v) for u, v in zip(got, new)) and not grads[:, Hq + Hk:].any()
    got = ts.ts_qk_rope_bwd(dq, dk, x, y, pos, r, wq, wk, dq=dq, dk=dk)
    assert got[0] is dq and all(same_bits(u, v) for u, v in zip(got, new))


@pytest.mark.parametrize("d", [64, 128])
def test_rope_of_rows_four_gigabytes_apart(d):
    say("far rows", d)
    T, H, stride = 9, 3, (1 << 29) + 8  # elements: the last row starts past 2^32
    g = rng(2)
    mem = torch.empty((T - 1) * stride + 2 * H * d, dtype=torch.bfloat16, device="cuda")
    q = mem.as_strided((T, H, d), (stride, d, 1))
    k = mem.as_strided((T, H, d), (stride, d, 1), H * d)
    q.copy_(normal(g, T, H, d))
    k.copy_(normal(g, T, H, d))
    pos = torch.randint(-(1 << 31), (1 << 31) - 1, (T, 3), generator=g, device="cuda").int()
    r = ts.rope(AXES[d], interleaved=False)
    near_q = rope_tol(q, None, R.angles(pos, r.freq, AXES[d]), False, 1e-6)
    near_k = rope_tol(k, None, R.angles(pos, r.freq, AXES[d]), False, 1e-6)
    got = ts.ts_qk_rope(q, k, pos, r, q_out=q)
    near("q", got[0], *near_q)
    near("k", got[1], *near_k)


def test_norm_at_the_ends_of_bfloat16():
    d, eps = 128, 1e-6
    top = torch.finfo(torch.bfloat16).max
    x = torch.randn(6, 2, d, generator=rng(3), device="cuda")
    x = x.sign() * (0.5 + 0.5 * x.abs().clamp(max=1))
    for i, size in enumerate((top, 1e30, 1e-30, 2.0 ** -133, 0.0, 1.0)):
        x[i] *= size
    x = x.bfloat16()
    w = torch.ones(d, device="cuda")
    for e in (eps, 2.0 ** -126, 1e30):
        got, _ = ts.ts_qk_rope(x, None, q_weight=w, eps=e)
        ref = x.double() / torch.sqrt(x.double().square().mean(-1, keepdim=True) + e)
        near("eps %g" % e, got, ref, R.HALF * ref.abs() + R.FINE * ref.abs() + 2.0 ** -133)
        dy = torch.randn(x.shape, generator=rng(4), device="cuda").bfloat16()
        dx, _, dw, _ = ts.ts_qk_rope_bwd(dy, None, x, None, q_weight=w, eps=e)
        want, want_w, mag, mag_w = R.rope_bwd(dy.double(), x.double(), w.double(), None, True, e)
        near("dx", dx, want, R.HALF * want.abs() + 1.01 * R.FINE * mag + 2.0 ** -126)
        near("dw", dw, want_w, R.FINE * mag_w)


def test_what_is_not_finite_stays_in_its_head():
    d = 64
    g = rng(5)
    x = normal(g, 5, 4, d).bfloat16()
    x[1, 2, 7], x[3, 0, 0], x[4, 3, 63] = math.inf, math.nan, -math.inf
    w, r, pos = torch.ones(d, device="cuda"), ts.rope(AXES[d]), torch.ones(5, 3, dtype=torch.int32, device="cuda")
    bad = torch.zeros(5, 4, dtype=torch.bool, device="cuda")
    bad[1, 2] = bad[3, 0] = bad[4, 3] = True
    for weight in (w, None):
        y, _ = ts.ts_qk_rope(x, None, pos, r, q_weight=weight)
        assert torch.equal(~y.isfinite().all(-1), bad)
        ref = R.rope(x.double(), None if weight is None else w.double(), R.angles(pos, r.freq, AXES[d]), True, 1e-6)
        assert torch.equal(ref.isnan(), y.double().isnan())
    dx, _, _, _ = ts.ts_qk_rope_bwd(normal(g, 5, 4, d).bfloat16(), None, x, None, pos, r, q_weight=w)
    assert torch.equal(~dx.isfinite().all(-1), bad)


@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("d", [64, 128])
def test_calls_larger_than_the_caches(d, interleaved):
    """More than 256 MB read and written, which go past the caches: bit for bit what the halves' calls give (but the weights'
    gradients, whose sums go by the sizes)."""
    say("large", d, interleaved)
    Hq, Hk = 20, 12
    T = (300 << 20) // ((Hq + Hk) * d * 4) + 1
    g = rng(45)
    q, k, dq, dk = (normal(g, T, H, d).bfloat16() for H in (Hq, Hk, Hq, Hk))
    wq, wk = 1 + 0.3 * normal(g, d), 1 + 0.3 * normal(g, d)
    r, pos = ts.rope(AXES[d], interleaved=interleaved), torch.randint(0, 99, (T, 3), generator=g, device="cuda").int()
    cut = T // 2
    parts = [slice(0, cut), slice(cut, T)]
    whole = ts.ts_qk_rope(q, k, pos, r, wq, wk)
    back = ts.ts_qk_rope_bwd(dq, dk, q, k, pos, r, wq, wk)
    mag = [torch.zeros(d, dtype=torch.double, device="cuda") for _ in range(2)]
    dw = [torch.zeros(d, dtype=torch.double, device="cuda") for _ in range(2)]
    for at in parts:
        got = ts.ts_qk_rope(q[at], k[at], pos[at], r, wq, wk)
        assert all(same_bits(a[at], b) for a, b in zip(whole, got))
        got = ts.ts_qk_rope_bwd(dq[at], dk[at], q[at], k[at], pos[at], r, wq, wk)
        assert all(same_bits(a[at], b) for a, b in zip(back[:2], got))
        for i, (dy, x, w) in enumerate(((dq, q, wq), (dk, k, wk))):
            _, part, _, m = R.rope_bwd(dy[at].double(), x[at].double(), w.double(), R.angles(pos[at], r.freq, AXES[d]), interleaved, 1e-6)
            dw[i] += part
            mag[i] += m
    for i in range(2):
        near("dw", back[2 + i], dw[i], R.FINE * mag[i])


def test_no_tokens():
    x = torch.zeros(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, device="cuda")
    q, k = ts.ts_qk_rope(x, x, q_weight=w)
    assert q.shape == k.shape == x.shape
    grads = [torch.full((64,), 7.0, device="cuda") for _ in range(2)]
    dq, dk, dw, dw2 = ts.ts_qk_rope_bwd(x, x, x, x, q_weight=w, k_weight=w, dq_weight=grads[0], dk_weight=grads[1])
    assert dw is grads[0] and not dw.any() and not dw2.any()


def test_rope_against_differences():
    """The gradients of a sum of the results, with the forward kernel itself in place of the formula: a difference of results rounded to
    bfloat16 is off by 2^-8 of each at most, 2 R.HALF |y| |dy| / h in all, beside the second order's h^2."""
    g = rng(6)
    d, T, h = 64, 3, 0.25
    x = (normal(g, T, 1, d)).bfloat16()
    w, r = 1 + 0.3 * normal(g, d), ts.rope(AXES[d])
    pos = torch.randint(0, 50, (T, 3), generator=g, device="cuda").int()
    dy = normal(g, T, 1, d).bfloat16()
    dx, _, dw, _ = ts.ts_qk_rope_bwd(dy, None, x, None, pos, r, q_weight=w)
    for i in (0, 9, 63):
        e = torch.zeros(d, device="cuda")
        e[i] = h
        up, down = (ts.ts_qk_rope(x, None, pos, r, q_weight=w + s * e)[0].double() for s in (1, -1))
        num = ((up - down) * dy.double()).sum().item() / (2 * h)  # linear in w: no second order
        slack = (R.HALF * (up.abs() + down.abs()) * dy.double().abs()).sum().item() / (2 * h)
        assert abs(num - dw[i].item()) <= slack and slack < 30


# ---- gradients of attention


@pytest.mark.parametrize("d", [64, 128])
def test_a_segment_s_bits_are_its_own(d):
    """With forced ranges, alone as in a batch, whatever the batch's tiles."""
    say("own bits", d)
    lq, lk, H = [700, 33, 1200, 0, 260], [900, 1000, 65, 40, 260], 3
    for n in (1, 3):
        args = attn_inputs(lq, lk, H, d, None, seed=7)
        got = ts.ts_attn_bwd(*args, num_splits=n)
        big = [2000] * 14  # so many that d = 128 takes its large tiles
        wide = attn_inputs(lq + big, lk + big, H, d, None, seed=8)
        for x, y in zip(wide[:6], args[:6]):
            x[:y.shape[0]] = y
        many = ts.ts_attn_bwd(*wide, num_splits=n)
        for a, b in zip(got, many):
            assert same_bits(a, b[:a.shape[0]])
        q, k = R.offsets(lq), R.offsets(lk)
        for s in range(len(lq)):
            cut = [x[a:b] for x, (a, b) in zip(args[:6], ((q[s], q[s + 1]), (q[s], q[s + 1]), (k[s], k[s + 1]), (k[s], k[s + 1]), (q[s], q[s + 1]),
                                                          (q[s], q[s + 1])))]
            cu = [torch.tensor([0, m], dtype=torch.int32, device="cuda") for m in (lq[s], lk[s])]
            one = ts.ts_attn_bwd(*cut, *cu, lq[s], lk[s], num_splits=n)
            for a, b in zip(one, (got[0][q[s]:q[s + 1]], got[1][k[s]:k[s + 1]], got[2][k[s]:k[s + 1]])):
                assert same_bits(a, b)


@pytest.mark.parametrize("d", [64, 128])
def test_memory_past_32_bits(d):
    """Tensors of 4.5 GB: the last segment against its own call."""
    say("past 32 bits", d)
    H, L = 40, 300
    n = int(4.5e9 / (2 * H * d * L))
    g = rng(9)
    q, k, v, d_o = (torch.empty(n * L, H, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(4))
    cu = torch.arange(0, n + 1, device="cuda").mul_(L).int()
    o, lse = ts.ts_attn_fwd_kvcache(q, k, v, cu, cu, L, L, return_lse=True)
    got = ts.ts_attn_bwd(d_o, q, k, v, o, lse, cu, cu, L, L, num_splits=1)
    at = slice((n - 1) * L, n * L)
    one = ts.ts_attn_bwd(*(x[at] for x in (d_o, q, k, v, o, lse)), cu[:2], cu[:2], L, L, num_splits=1)
    assert all(same_bits(a, b[at]) for a, b in zip(one, got))
    ref, tol = R.packed_attn_bwd(*(x[at][:, :2].double() for x in (d_o, q, k, v, o, lse)), [0, L], [0, L], ts.default_scale(d))
    for name, x, y, t in zip(("dq", "dk", "dv"), one, ref, tol):
        near(name, x[:, :2], y, t)


@pytest.mark.parametrize("splits", [0, 1, 2])
@pytest.mark.parametrize("d", [64, 128])
def test_more_segments_than_the_plan_sorts(d, splits):
    say("many segments", d, splits)
    g = np.random.default_rng(46)
    lq, lk = ([int(x) for x in g.integers(0, 40, 700)] for _ in range(2))
    lq[300], lk[301], lk[699] = 150, 290, 129
    args = attn_inputs(lq, lk, 2, d, None, seed=46)
    got = ts.ts_attn_bwd(*args, num_splits=splits)
    check_attn(lq, lk, 2, d, ts.default_scale(d), got, args)


@pytest.mark.parametrize("d", [64, 128])
def test_longest_lengths_that_are_only_bounds(d):
    """Maxima far above the lengths, as a program that does not read its offsets states them: more workgroups are started than
    have work, and of forced ranges the bits are the same."""
    say("bounds", d)
    lq, lk = [130, 0, 700, 1], [200, 40, 333, 1]
    args = attn_inputs(lq, lk, 3, d, None, seed=47)
    want = ts.ts_attn_bwd(*args, num_splits=2)
    got = ts.ts_attn_bwd(*args[:8], 5000, 70000, num_splits=2)
    assert all(same_bits(a, b) for a, b in zip(got, want))
    check_attn(lq, lk, 3, d, ts.default_scale(d), ts.ts_attn_bwd(*args[:8], 5000, 70000), args)


BAD = [  # cu_q, cu_k, for 150 queries and 400 keys, at most 100 and 400 of a segment
    ([1, 100, 150], [0, 0, 400]), ([0, 101, 150], [0, 0, 400]), ([0, 100, 149], [0, 0, 400]), ([0, -5, 150], [0, 0, 400]),
    ([0, 100, 151], [0, 0, 400]), ([0, 100, 150], [0, 401, 400]), ([0, 100, 150], [0, 10, 9]), ([0, 100, 150], [5, 10, 400]),
    ([0, 120, 90], [0, 0, 400]), ([0, -2147483648, 2147483647], [0, 0, 400]),
]


@pytest.mark.parametrize("splits", [0, 2])
@pytest.mark.parametrize("cu", BAD, ids=str)
def test_offsets_that_break_the_rules_leave_the_gradients_alone(cu, splits):
    say("bad offsets", cu, splits)
    q, k = torch.ones(150, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(400, 2, 64, dtype=torch.bfloat16, device="cuda")
    outs = [torch.full_like(x, 7.0) for x in (q, k, k)]
    cq, ck = (torch.tensor(c, dtype=torch.int32, device="cuda") for c in cu)
    ts.ts_attn_bwd(q, q, k, k, q, torch.zeros(150, 2, device="cuda"), cq, ck, 100, 400, dq=outs[0], dk=outs[1], dv=outs[2], num_splits=splits)
    torch.cuda.synchronize()
    assert all(bool((x == 7.0).all()) for x in outs)


def test_validation_mode_names_them(monkeypatch):
    monkeypatch.setenv("TS_ATTN_VALIDATE", "1")
    args = attn_inputs([100, 50], [0, 400], 2, 64, None, seed=10)
    ts.ts_attn_bwd(*args)
    for cu, at in ((torch.tensor([0, 101, 150]), 6), (torch.tensor([0, 0, 399]), 7)):
        bad = list(args)
        bad[at] = cu.int().cuda()
        with pytest.raises(ts.TsAttnError) as e:
            ts.ts_attn_bwd(*bad)
        assert e.value.status == 10


@pytest.mark.parametrize("d", [64, 128])
def test_keys_that_no_query_sees(d):
    """A key of score -infinity for every query has a weight of 0: dk and dv are 0 there and finite elsewhere; dq is 0 times
    infinity in that channel, as the formula has it.  Ragged ends beside it."""
    lq, lk, H = [77, 130], [93, 190], 2
    g = rng(11)
    q, v, d_o = (normal(g, sum(n), H, d).bfloat16() for n in (lq, lk, lq))
    k = normal(g, sum(lk), H, d).bfloat16()
    q[..., 3] = q[..., 3].abs() + 0.5
    k[50, :, 3] = -math.inf
    k[200, 1, 3] = -math.inf
    cu_q, cu_k = (torch.tensor(R.offsets(n), dtype=torch.int32, device="cuda") for n in (lq, lk))
    o, lse = R.packed_attn(*(x.double() for x in (q, k, v)), R.offsets(lq), R.offsets(lk), ts.default_scale(d))
    o, lse = o.bfloat16(), lse.float()
    assert bool(o.isfinite().all()) and bool(lse.isfinite().all())
    dq, dk, dv = ts.ts_attn_bwd(d_o, q, k, v, o, lse, cu_q, cu_k, max(lq), max(lk))
    clean = torch.where(k.isinf(), torch.tensor(-3e4, device="cuda", dtype=k.dtype), k)  # (as good as -infinity)
    ref, tol = R.packed_attn_bwd(*(x.double() for x in (d_o, q, clean, v, o, lse)), R.offsets(lq), R.offsets(lk), ts.default_scale(d))
    near("dk", dk, ref[1], tol[1])
    near("dv", dv, ref[2], tol[2])
    assert not dk[50].any() and not dv[50].any() and not dk[200, 1].any()
    nan = torch.zeros_like(dq, dtype=torch.bool)
    nan[:77, :, 3] = True
    nan[77:, 1, 3] = True
    assert torch.equal(dq.isnan(), nan)
    near("dq", torch.where(nan, 0, dq), torch.where(nan, 0, ref[0]), tol[0])


def test_nan_stays_in_its_segment_and_head():
    lq, lk, H, d = [40, 300], [70, 257], 2, 64
    args = list(attn_inputs(lq, lk, H, d, None, seed=12))
    want = ts.ts_attn_bwd(*args, num_splits=1)
    args[0] = args[0].clone()
    args[0][13, 1, 5] = math.nan  # d_o of one query
    got = ts.ts_attn_bwd(*args, num_splits=1)
    nq, nk = torch.zeros(340, 2, d, dtype=torch.bool, device="cuda"), torch.zeros(327, 2, d, dtype=torch.bool, device="cuda")
    nq[13, 1] = True
    nk[:70, 1] = True
    assert torch.equal(got[0].isnan(), nq) and torch.equal(got[1].isnan(), nk)
    nv = torch.zeros_like(nk)
    nv[:70, 1, 5] = True
    assert torch.equal(got[2].isnan(), nv)
    for a, b, n in zip(got[1:], want[1:], (nk, nv)):
        assert same_bits(a[~n], b[~n])
    assert same_bits(got[0][40:], want[0][40:]) and same_bits(got[0][:, 0], want[0][:, 0])
    # in its own tile a neighbour may keep its rounding's common part, within the same tolerance
    clean = [x.clone() for x in args[:6]]
    clean[0][13, 1] = 0
    ref, tol = R.packed_attn_bwd(*(x.double() for x in clean), R.offsets(lq), R.offsets(lk), ts.default_scale(d))
    near("dq", torch.where(nq, 0, got[0]), torch.where(nq, 0, ref[0]), tol[0])


def test_large_and_small_scores():
    """Weights of 0 and of 1: one key takes a row, whose gradient then is rounding alone."""
    for spread in (8.0, 1e-20):
        for d in (64, 128):
            lq, lk = [130, 64], [200, 333]
            args = attn_inputs(lq, lk, 2, d, 0.5, seed=13, spread=spread)
            got = ts.ts_attn_bwd(*args, scale=0.5)
            check_attn(lq, lk, 2, d, 0.5, got, args)


def test_attention_against_differences():
    """The gradient of sum(o d_o) along a direction u, with the forward kernel in place of the formula.  Each result is rounded by HALF of
    itself and has weights rounded by HALF: 2 HALF |o| |d_o| at most on each side, with steps so large that this leaves something, and
    so small that the third order does not count (u is a twentieth of q)."""
    g = rng(14)
    lq, lk, H, d = [64], [40], 2, 64
    args = attn_inputs(lq, lk, H, d, None, seed=14)
    d_o, q, k, v, o, lse, cu_q, cu_k, mq, mk = args
    dq, dk, dv = ts.ts_attn_bwd(*args)
    for at, x, grad in ((0, q, dq), (1, k, dk), (2, v, dv)):
        u = grad.float() / grad.float().square().mean().sqrt() * 0.1  # along the gradient, where the difference is largest
        sides = []
        for s in (1, -1):
            y = [q, k, v]
            y[at] = (x.float() + s * u).bfloat16()
            sides.append((y[at], ts.ts_attn_fwd_kvcache(*y, cu_q, cu_k, mq, mk)))
        num = ((sides[0][1].double() - sides[1][1].double()) * d_o.double()).sum().item()
        want = ((sides[0][0].double() - sides[1][0].double()) * grad.double()).sum().item()
        noise = (2 * R.HALF * (sides[0][1].double().square() + sides[1][1].double().square()) * d_o.double().square()).sum().sqrt().item()
        say("difference %.4f, gradient %.4f, noise %.4f" % (num, want, noise))
        assert abs(num - want) <= noise + 0.05 * abs(want) and abs(want) > 4 * noise


@pytest.mark.parametrize("d", [64, 128])
def test_keys_that_have_much_in_common(d):
    """Keys in which a few channels stand far out, all to one side, as a trained model's do: rounding S makes dq off by its error times
    what they have in common, unless that is taken off again.  With it dq is off by its own rounding (0.0017 of its norm,
    rms of HALF / sqrt(3) at most) and that of S times the keys' spread, as much again: 0.0032 at most where every element of either is at
    the low end of its binade, 0.0024 on average; 0.0030 leaves room for some.  Uncorrected, with 8 times the spread, it is 0.013."""
    lq, lk, H = [300, 500], [1000, 700], 3
    args = list(attn_inputs(lq, lk, H, d, None, seed=16))
    q, k, v = args[1:4]
    k = (normal(rng(17), *k.shape) + 8 * normal(rng(18), H, d).sign()).bfloat16()
    q = (q.float() * 0.3).bfloat16()  # (scores of a sensible spread: a constant added to a row's scores does not matter)
    o, lse = ts.ts_attn_fwd_kvcache(q, k, v, *args[6:], return_lse=True)
    got = ts.ts_attn_bwd(args[0], q, k, v, o, lse, *args[6:])
    ref, tol = R.packed_attn_bwd(*(x.double() for x in (args[0], q, k, v, o, lse)), R.offsets(lq), R.offsets(lk), ts.default_scale(d))
    for name, x, y, t in zip(("dq", "dk", "dv"), got, ref, tol):
        near(name, x, y, t)
        off = ((x.double() - y).norm() / y.norm()).item()
        say(name, "off by %.4f" % off)
        assert off < 0.0030


# ---- graphs and streams


def test_a_captured_training_step_replays():
    g = rng(15)
    T, H, d = 300, 4, 64
    cu, mx = torch.tensor([0, 100, 300], dtype=torch.int32, device="cuda"), 200
    q, k, v, d_o = (normal(g, T, H, d).bfloat16() for _ in range(4))
    w = 1 + 0.2 * normal(g, d)
    r, pos = ts.rope(AXES[d]), torch.randint(0, 30, (T, 3), generator=g, device="cuda").int()

    def step():
        a, b = ts.ts_qk_rope(q, k, pos, r, w, w)
        o, lse = ts.ts_attn_fwd_kvcache(a, b, v, cu, cu, mx, mx, return_lse=True, num_splits=1)
        da, db, dv = ts.ts_attn_bwd(d_o, a, b, v, o, lse, cu, cu, mx, mx)
        return (*ts.ts_qk_rope_bwd(da, db, q, k, pos, r, w, w), dv)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):  # two graphs live at once
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        graphs.append((graph, out))
    for i in range(4):
        for x in (q, k, v, d_o):
            x.copy_(normal(g, T, H, d))
        want = step()
        for graph, out in graphs:
            graph.replay()
        eager = step()  # beside the replays
        torch.cuda.synchronize()
        for out in (graphs[0][1], graphs[1][1], eager):
            assert all(same_bits(a, b) for a, b in zip(out, want)), "replay %d" % i


def test_two_streams_at_once():
    jobs = []
    for i in range(2):
        s = torch.cuda.Stream()
        lq = [1500 + 100 * i, 64]
        jobs.append((s, attn_inputs(lq, lq, 3, 128 if i else 64, None, seed=20 + i)))
    want = [ts.ts_attn_bwd(*a) for _, a in jobs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, (s, a) in enumerate(jobs):
            with torch.cuda.stream(s):
                got[i].append(ts.ts_attn_bwd(*a))
    torch.cuda.synchronize()
    for i in range(2):
        for x in got[i]:
            assert all(same_bits(a, b) for a, b in zip(x, want[i]))


# ---- together


@pytest.mark.parametrize("d", [64, 128])
def test_a_training_step(d):
    """Norm and rotation, attention, and back: each call against the formula on what it was given, and the whole against automatic
    differentiation in 64 bits.  That has no roundings in between: q', k' and o are off by HALF, P and S and the gradients that
    pass from call to call by HALF again, each independent of the others; of gradients that are sums of many terms 6 such are off by
    sqrt(6) HALF / sqrt(3) = 0.0055 (rms), and 0.02 is more than three times that."""
    g = rng(30 + d)
    lens, H = [130, 1, 257], 3
    T, cu = sum(lens), torch.tensor(R.offsets(lens), dtype=torch.int32, device="cuda")
    rows = normal(g, T, 3 * H, d).bfloat16()
    q, k, v = rows[:, :H], rows[:, H:2 * H], rows[:, 2 * H:].contiguous()
    wq, wk = 1 + 0.3 * normal(g, d), 1 + 0.3 * normal(g, d)
    r, pos = ts.rope(AXES[d]), torch.stack([torch.arange(T) // 100, torch.arange(T) // 10 % 10, torch.arange(T) % 10], 1).int().cuda()
    d_o = normal(g, T, H, d).bfloat16()
    scale = ts.default_scale(d)
    a, b = ts.ts_qk_rope(q, k, pos, r, wq, wk)
    o, lse = ts.ts_attn_fwd_kvcache(a, b, v, cu, cu, max(lens), max(lens), return_lse=True)
    da, db, dv = ts.ts_attn_bwd(d_o, a, b, v, o, lse, cu, cu, max(lens), max(lens))
    dq, dk, dwq, dwk = ts.ts_qk_rope_bwd(da, db, q, k, pos, r, wq, wk)
    check_attn(lens, lens, H, d, scale, (da, db, dv), (d_o, a, b, v, o, lse))
    leaves = [x.double().requires_grad_() for x in (q, k, v, wq, wk)]
    angle = R.angles(pos, r.freq, AXES[d])
    x, y = (R.rope(leaves[i], leaves[3 + i], angle, True, 1e-6) for i in range(2))
    outs = torch.cat([torch.stack([R.attn(x[s:e, h], y[s:e, h], leaves[2][s:e, h], scale)[0] for h in range(H)], 1)
                      for s, e in zip(R.offsets(lens)[:-1], R.offsets(lens)[1:])])
    want = torch.autograd.grad(outs, leaves, d_o.double())
    for name, got, ref in zip(("dq", "dk", "dv", "dwq", "dwk"), (dq, dk, dv, dwq, dwk), want):
        off = ((got.double() - ref).norm() / ref.norm()).item()
        say(name, "off by %.4f" % off)
        assert off < 0.02


def test_a_serving_step():
    """One token each of three sessions: norm and rotation at its place in the stream, into the session's 8-bit cache, and
    attention over it.  Cached keys are within half an e4m3 step of the formula's, and attention is over exactly them."""
    d, H, G = 128, 2, 3
    g = rng(40)
    lens0, pages = [70, 0, 129], 8
    cache = ts.session_cache(pages, H, d)
    table = torch.tensor([[0, 1, 2], [3, 4, 5], [6, 7, -1]], dtype=torch.int32, device="cuda")[[0, 1, 0]].clone()
    table[2] = torch.tensor([5, 6, 7])
    r, w = ts.rope(AXES[d]), 1 + 0.2 * normal(g, d)
    lens = torch.zeros(3, dtype=torch.int32, device="cuda")
    keys, values = [[], [], []], [[], [], []]

    def step(counts):
        nonlocal lens
        n = sum(counts)
        q, k, v = normal(g, n, H * G, d).bfloat16(), normal(g, n, H, d).bfloat16(), normal(g, n, H, d).bfloat16()
        at = torch.cat([torch.arange(c, device="cuda") + l for c, l in zip(counts, lens.tolist())])
        pos = torch.stack([at // 60, at // 10 % 6, at % 10], 1).int()
        cu = torch.tensor(R.offsets(counts), dtype=torch.int32, device="cuda")
        a, b = ts.ts_qk_rope(q, k, pos, r, w, w)
        lens = ts.ts_cache_append(cache, b, v, cu, max(counts), table, lens)
        ref = R.rope(k.double(), w.double(), R.angles(pos, r.freq, AXES[d]), True, 1e-6)
        for s in range(3):
            keys[s].append(ref[cu[s]:cu[s + 1]])
        o = ts.ts_cache_attn(a, cache, cu, max(counts), table, lens, 192)
        return a, o, cu

    step(lens0)
    a, o, cu = step([1, 1, 1])
    assert lens.tolist() == [71, 1, 130]
    kf = (cache.k.float() * torch.exp2(cache.k_exp.float() - 127)[:, :, None, None]).double()
    vf = (cache.v.float() * torch.exp2(cache.v_exp.float() - 127)[:, :, None, None]).double()
    for s in range(3):
        n = lens[s].item()
        want = torch.cat(keys[s])
        rows = [table[s, j // 64].item() for j in range(n)]
        got = torch.stack([kf[p, :, j % 64] for j, p in enumerate(rows)])
        val = torch.stack([vf[p, :, j % 64] for j, p in enumerate(rows)])
        least = torch.stack([torch.exp2(cache.k_exp[p].double() - 127 - 10) for p in rows])[:, :, None]  # half the smallest step, 2^-9
        # rounded to bfloat16, then to e4m3 (twice, where a page's exponent rose)
        near("keys", got, want, (2 * 2.0 ** -4 + R.HALF) * 1.1 * want.abs() + 2.1 * least)
        for h in range(H * G):
            ref, _ = R.attn(a[s:s + 1, h].double(), got[:, h // G], val[:, h // G], ts.default_scale(d))
            off = (o[s:s + 1, h].double() - ref).abs().max().item()
            assert off <= 2e-2, off


# ---- workspaces of the C calls


@pytest.mark.parametrize("d", [64, 128])
def test_a_smaller_workspace_divides_the_work_less(d):
    """From the least that the call takes to more than it makes use of: the gradients hold, and what lies behind the stated bytes stays as it
    is, as the gradients' neighbours do."""
    say("workspace", d)
    lib = ts.load_block()
    lq, lk, H = [300, 70], [1500, 900], 2
    args = attn_inputs(lq, lk, H, d, None, seed=50)
    sizes = (2, 300, 1500, 370, 2400, H, d)
    most, least = (lib.ts_attn_bwd_workspace(*sizes, n) for n in (0, 1))
    assert 0 < least < most
    room = 4096
    for given in (least, (least + most) // 2 // 256 * 256, most, most + 65536):
        work = torch.full((given + room,), 0xA5, dtype=torch.uint8, device="cuda")
        outs = [torch.full((x.shape[0] + 2, H, d), 7.0, dtype=torch.bfloat16, device="cuda") for x in (args[1], args[2], args[3])]
        rc = lib.ts_attn_bwd(*(x.data_ptr() for x in args[:6]), *(x[1:].data_ptr() for x in outs), *(x.data_ptr() for x in args[6:8]), *sizes,
                             ts.default_scale(d), 0, work.data_ptr(), given, torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        check_attn(lq, lk, H, d, ts.default_scale(d), [x[1:-1] for x in outs], args)
        assert bool((work[given:] == 0xA5).all())
        assert all(bool((x[[0, -1]] == 7.0).all()) for x in outs)
    assert lib.ts_attn_bwd(*(x.data_ptr() for x in args[:6]), *(x[1:].data_ptr() for x in outs), *(x.data_ptr() for x in args[6:8]), *sizes,
                           ts.default_scale(d), 0, work.data_ptr(), least - 1, torch.cuda.current_stream().cuda_stream) == 13  # TS_ERR_SCRATCH
