"""The attention calls with keys whose scores are -infinity (a channel of -infinity in the key, of one sign in every query): they have a
weight of 0, wherever they lie and whatever the tile, and change nothing else."""
import math

import pytest
import torch

import block_ref as R
from test_gpu_block import near, normal, rng, same_bits, say

pytestmark = pytest.mark.gpu

ts = pytest.importorskip("paper_2606_19271_amd")


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ts.load()
    ts.load_block()


def inputs(lq, lk, H, d, hidden, seed):
    """hidden: rows of k."""
    g = rng(seed)
    q, k, v = (normal(g, sum(n), H, d).bfloat16() for n in (lq, lk, lk))
    q[..., 3] = q[..., 3].abs() + 0.5
    k[list(hidden), :, 3] = -math.inf
    return q, k, v


def definition(q, k, v, lq, lk, scale):
    """o and lse in 64 bits and how far each may be off.  Weights are rounded to bfloat16, HALF of each one way or the other, and divided by
    the sum of the rounded ones: o is off by sum p_j e_j (v_j - o), |e_j| <= HALF, in one of 10^7 cases by 6 sqrt(sum (p_j (v_j -
    o))^2) HALF, and rounded once more; lse by sum p_j e_j.  Scores, and their difference to the maximum, are sums in 32 bits."""
    o, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=q.dtype, device=q.device)
    tol_o, tol_l = torch.zeros_like(q), torch.zeros_like(lse)
    for a, b, c, e in R.segments(R.offsets(lq), R.offsets(lk)):
        for h in range(q.shape[1]):
            x, y, w = q[a:b, h], k[c:e, h], v[c:e, h]
            s = scale * (x @ y.T)
            some = (s != -math.inf).any(1)
            p = torch.softmax(s, 1)[some]
            seen = torch.where(y.isinf(), 0, y)
            arg = R.FINE * (scale * (x[some].abs() @ seen.abs().T) + torch.logsumexp(s[some], 1).abs()[:, None] + 1)
            far = (w[None] - (p @ w)[:, None]).abs()  # [rows, keys, d]
            sums = torch.minimum((p[..., None] * far).sum(1), 6 * (p[..., None] * far).square().sum(1).sqrt())
            fine = ((p * arg)[..., None] * far).sum(1) + R.FINE * (p @ w.abs())
            out, tol = torch.zeros_like(x), torch.zeros_like(x)
            out[some], tol[some] = p @ w, R.HALF * (p @ w).abs() + (1 + R.HALF) * (R.HALF * sums + fine) + R.LEAST
            o[a:b, h], tol_o[a:b, h] = out, tol
            lse[a:b, h] = torch.where(some, torch.logsumexp(s, 1), -math.inf)
            t = torch.zeros(b - a, dtype=q.dtype, device=q.device)
            t[some] = R.HALF * torch.clamp(6 * p.square().sum(1).sqrt(), max=1) + (p * arg).sum(1) + R.FINE * (1 + torch.logsumexp(s[some], 1).abs())
            tol_l[a:b, h] = t
    return o, lse, tol_o, tol_l


def close(name, o, lse, want):
    ref_o, ref_l, tol_o, tol_l = want
    near(name + " o", o, ref_o, tol_o)
    if lse is None:
        return
    empty = ref_l == -math.inf
    assert torch.equal(lse == -math.inf, empty) and not lse.isnan().any()
    near(name + " lse", torch.where(empty, 0, lse), torch.where(empty, 0, ref_l), tol_l)


# lengths that end in tiles of 2 to 63 rows, in every kind of tile; 258 and 513 leave thin ones
SIZES = [([130], [190], 2), ([77, 130], [93, 190], 2), ([300], [500], 2), ([1000], [700], 2), ([2], [500], 2), ([258, 1, 40], [300, 70, 200], 2),
         ([513, 100, 33], [130, 600, 64], 40), ([700] * 3, [333] * 3, 40)]


def places(which, lk):
    """Rows of all segments' keys that are hidden."""
    at, rows = 0, []
    for n in lk:
        part = {"one": [n // 2], "first": range(min(n - 1, 64)), "two tiles": range(min(n - 1, 256)), "even": range(0, n - 1, 2), "last": range(n - 40, n),
                "all but the last": range(n - 1), "all": range(n)}[which]
        rows += [at + i for i in part if i >= 0]
        at += n
    return rows


@pytest.mark.parametrize("splits", [0, 1, 3])
@pytest.mark.parametrize("which", ["one", "first", "two tiles", "even", "last", "all but the last", "all"])
@pytest.mark.parametrize("d", [64, 128])
def test_chunks(d, which, splits):
    for i, (lq, lk, H) in enumerate(SIZES):
        say("chunk", lq, lk, H, d, which, splits)
        q, k, v = inputs(lq, lk, H, d, places(which, lk), 80 + i)
        cu_q, cu_k = (torch.tensor(R.offsets(n), dtype=torch.int32, device="cuda") for n in (lq, lk))
        o, lse = ts.ts_attn_fwd_kvcache(q, k, v, cu_q, cu_k, max(lq), max(lk), return_lse=True, num_splits=splits)
        h = slice(0, 2)
        close("chunk", o[:, h], lse[:, h], definition(*(x[:, h].double() for x in (q, k, v)), lq, lk, ts.default_scale(d)))


@pytest.mark.parametrize("which", ["one", "first", "even", "all"])
@pytest.mark.parametrize("d", [64, 128])
def test_packed_and_dense(d, which):
    for i, (lens, H) in enumerate((([130, 77, 300], 2), ([520, 33, 1000], 20), ([333] * 4, 2), ([333] * 4, 40))):
        say("packed", lens, H, d, which)
        q, k, v = inputs(lens, lens, H, d, places(which, lens), 90 + i)
        cu = torch.tensor(R.offsets(lens), dtype=torch.int32, device="cuda")
        want = definition(*(x[:, :2].double() for x in (q, k, v)), lens, lens, ts.default_scale(d))
        close("packed", ts.ts_attn_fwd_varlen(q, k, v, cu, max(lens))[:, :2], None, want)
        if len(set(lens)) == 1:
            x = [y.view(len(lens), lens[0], H, d) for y in (q, k, v)]
            close("dense", ts.ts_attn_fwd(*x).view_as(q)[:, :2], None, want)


@pytest.mark.parametrize("d", [64, 128])
def test_a_row_that_is_not_finite_says_so(d):
    """A query of NaN, and one that meets a key of +infinity: NaN results and a NaN log-sum-exp, with and without ranges; whoever
    shares a tile with it has its own result or NaN, never another number."""
    lq, lk, H = [70, 300], [130, 400], 2
    q, k, v = inputs(lq, lk, H, d, [20, 200], 95)
    clean = definition(*(x.double() for x in (q, k, v)), lq, lk, ts.default_scale(d))
    q = q.clone()
    q[5, 1, 7] = math.nan
    q[100, 0, 3] = -q[100, 0, 3]  # (key 200 is +infinity to it)
    bad = torch.zeros(370, H, dtype=torch.bool, device="cuda")
    bad[5, 1] = bad[100, 0] = True
    cu_q, cu_k = (torch.tensor(R.offsets(n), dtype=torch.int32, device="cuda") for n in (lq, lk))
    for splits in (0, 1, 2):
        o, lse = ts.ts_attn_fwd_kvcache(q, k, v, cu_q, cu_k, 300, 400, return_lse=True, num_splits=splits)
        assert o[bad].isnan().all() and lse[bad].isnan().all()
        also = lse.isnan() & ~bad
        assert also.sum() <= 2 and torch.equal(o.isnan().all(-1), bad | also)
        fine = ~(bad | also)
        near("o", o[fine], clean[0][fine], clean[2][fine])
        near("lse", lse[fine], clean[1][fine], clean[3][fine])


@pytest.mark.parametrize("d", [64, 128])
def test_rows_past_the_end_are_nobody_s(d):
    """The same queries in a tile of their own and ahead of another segment's: the same bits."""
    lq, lk, H = [45], [333], 2
    q, k, v = inputs(lq, lk, H, d, [7, 140], 96)
    cu = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 45], [0, 333], [0, 45, 90], [0, 333, 666])]
    one = ts.ts_attn_fwd_kvcache(q, k, v, cu[0], cu[1], 45, 333, return_lse=True, num_splits=1)
    q2, k2, v2 = (torch.cat([x, torch.full_like(x, math.nan)]) for x in (q, k, v))
    two = ts.ts_attn_fwd_kvcache(q2, k2, v2, cu[2], cu[3], 45, 333, return_lse=True, num_splits=1)
    assert all(same_bits(a, b[:45]) for a, b in zip(one, two)) and one[1].isfinite().all()


@pytest.mark.parametrize("splits", [0, 1, 3])
@pytest.mark.parametrize("scale", [None, -0.1])
@pytest.mark.parametrize("d", [64, 128])
def test_gradients_of_queries_that_see_nothing(d, scale, splits):
    """A log-sum-exp of -infinity, as the forward calls give it where all scores are, or as a caller marks rows with it: the row takes part
    in nothing.  In a segment whose keys all are hidden dk and dv are 0, and dq but in the hiding channel, where it is 0 times
    infinity; rows that the caller marks have dq = 0 and leave the others' gradients as they are without them."""
    say("see nothing", d, scale, splits)
    lq, lk, H = [130, 77, 40], [190, 93, 300], 2
    q, k, v = inputs(lq, lk, H, d, range(190, 283), 97)
    if scale is not None:
        q[..., 3] = -q[..., 3]
    d_o = normal(rng(98), sum(lq), H, d).bfloat16()
    cu_q, cu_k = (torch.tensor(R.offsets(n), dtype=torch.int32, device="cuda") for n in (lq, lk))
    o, lse = ts.ts_attn_fwd_kvcache(q, k, v, cu_q, cu_k, 130, 300, scale=scale, return_lse=True)
    assert (lse[130:207] == -math.inf).all() and not o[130:207].any() and lse[:130].isfinite().all() and lse[207:].isfinite().all()
    marked = [5, 100, 129, 210]
    o, lse = o.clone(), lse.clone()
    o[marked], lse[marked] = 0, -math.inf
    dq, dk, dv = ts.ts_attn_bwd(d_o, q, k, v, o, lse, cu_q, cu_k, 130, 300, scale=scale, num_splits=splits)
    assert not dk[190:283].any() and not dv[190:283].any() and dq[130:207, :, 3].isnan().all()
    dq = dq.clone()
    dq[130:207, :, 3] = 0
    assert not dq[130:207].any() and not dq[marked].any()
    use = ts.default_scale(d) if scale is None else scale
    keep = torch.ones(sum(lq), dtype=torch.bool, device="cuda")
    keep[marked] = keep[130:207] = False
    for a, b, c, e in ((0, 130, 0, 190), (207, 247, 283, 583)):
        rows = [x[a:b][keep[a:b]].double() for x in (d_o, q, o, lse)]
        for h in range(H):
            ref, tol = R.attn_bwd(rows[0][:, h], rows[1][:, h], k[c:e, h].double(), v[c:e, h].double(), rows[2][:, h], rows[3][:, h], use)
            for name, x, y, t in zip(("dq", "dk", "dv"), (dq[a:b, h][keep[a:b]], dk[c:e, h], dv[c:e, h]), ref, tol):
                near(name, x, y, t)
