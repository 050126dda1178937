"""The transformer block's calls (include/ts_block.h) on the GPU against their plain 64-bit forms (tests/block_ref.py)."""
import math

import numpy as np
import pytest
import torch

import block_ref as R

pytestmark = pytest.mark.gpu

ts = pytest.importorskip("paper_2606_19271_amd")

AXES = {64: (12, 10, 10), 128: (22, 21, 21)}


def say(*a):
    print("[gpu-test]", *a, flush=True)


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ts.load()
    ts.load_block()


def rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def near(name, got, ref, tol):
    """Every element within its tolerance."""
    off = (got.double() - ref).abs()
    bad = ~(off <= tol)
    worst = (off / tol.clamp(min=1e-300)).nan_to_num(math.inf).max().item() if off.numel() else 0.0
    say(name, "worst %.3f of its tolerance" % worst)
    assert not bad.any(), "%s: %d of %d elements off, first at %s: %r for %r, tolerance %r" % (
        name, bad.sum().item(), bad.numel(), bad.nonzero()[0].tolist(), got[bad][0].item(), ref[bad][0].item(), tol[bad][0].item())


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.int16 if a.element_size() == 2 else torch.int32),
                       b.contiguous().view(torch.int16 if b.element_size() == 2 else torch.int32))


# ---- norm and rotation


def rope_inputs(T, Hq, Hk, d, norm, turn, interleaved, fused, far, seed):
    g = rng(seed)
    if fused:
        rows = (normal(g, T, Hq + 2 * Hk, d) * 2).bfloat16()
        q, k = rows[:, :Hq], rows[:, Hq:Hq + Hk]
    else:
        q, k = (normal(g, T, Hq, d) * 2).bfloat16(), (normal(g, T, Hk, d) + 1).bfloat16() if Hk else None
    wq, wk = (1 + 0.3 * normal(g, d), 1 + 0.3 * normal(g, d)) if norm else (None, None)
    rope = pos = None
    if turn:
        rope = ts.rope(AXES[d], interleaved=interleaved)
        pos = torch.randint(-far - 1, far + 1, (T, 3), generator=g, device="cuda").int()
    return q, k, pos, rope, wq, wk if Hk else None


ROPE = [  # T, Hq, Hk, d, norm, turn, interleaved, fused, far
    (1, 1, 1, 64, True, True, True, False, 0),
    (1, 40, 8, 128, True, True, True, False, (1 << 31) - 1),
    (3, 7, 1, 128, True, True, False, True, 1000),
    (5, 2, 0, 64, True, True, False, False, 100),
    (257, 12, 12, 128, True, True, True, True, 5000000),
    (1001, 24, 12, 64, True, True, False, True, 100),
    (777, 12, 12, 128, False, True, True, False, 1000),
    (333, 5, 3, 64, False, True, False, True, 1000),
    (100, 9, 17, 128, True, False, True, True, 0),
    (4000, 40, 40, 128, True, True, True, True, 100),
]


@pytest.mark.parametrize("case", ROPE, ids=str)
def test_rope(case):
    T, Hq, Hk, d, norm, turn, interleaved, fused, far = case
    say("rope", case)
    q, k, pos, rope, wq, wk = rope_inputs(*case, seed=1)
    got = ts.ts_qk_rope(q, k, pos, rope, wq, wk, eps=1e-6)
    angle = R.angles(pos, rope.freq, AXES[d]) if turn else None
    for name, x, w, y in (("q", q, wq, got[0]), ("k", k, wk, got[1])):
        if x is None:
            assert y is None
            continue
        assert y.shape == x.shape and y.is_contiguous()
        w = None if w is None else w.double()
        ref, mag = (f(x.double(), w, angle, interleaved, 1e-6) for f in (R.rope, R.rope_slack))
        near(name, y, ref, R.HALF * ref.abs() + 1.01 * R.FINE * mag)


ROPE_BWD = [c for c in ROPE if c[0] > 1] + [(1, 2, 2, 128, True, True, True, False, 10), (20000, 3, 2, 64, True, True, True, True, 10)]


@pytest.mark.parametrize("case", ROPE_BWD, ids=str)
def test_rope_bwd(case):
    T, Hq, Hk, d, norm, turn, interleaved, fused, far = case
    say("rope_bwd", case)
    q, k, pos, rope, wq, wk = rope_inputs(*case, seed=2)
    g = rng(3)
    dq, dk = normal(g, T, Hq, d).bfloat16(), normal(g, T, Hk, d).bfloat16() if Hk else None
    got = ts.ts_qk_rope_bwd(dq, dk, q, k, pos, rope, wq, wk, eps=1e-6)
    again = ts.ts_qk_rope_bwd(dq, dk, q, k, pos, rope, wq, wk, eps=1e-6)
    angle = R.angles(pos, rope.freq, AXES[d]) if turn else None
    for i, (dy, x, w) in enumerate(((dq, q, wq), (dk, k, wk))):
        if dy is None:
            assert got[i] is None and got[2 + i] is None
            continue
        dx, dw, mag, mag_w = R.rope_bwd(dy.double(), x.double(), None if w is None else w.double(), angle, interleaved, 1e-6)
        near("dx", got[i], dx, R.HALF * dx.abs() + 1.01 * R.FINE * mag)
        assert same_bits(got[i], again[i])
        if w is None:
            assert got[2 + i] is None
        else:
            near("dw", got[2 + i], dw, R.FINE * mag_w)
            assert same_bits(got[2 + i], again[2 + i])


# ---- gradients of attention


def attn_inputs(lq, lk, H, d, scale, seed, spread=1.0):
    g = rng(seed)
    q, v, d_o = ((normal(g, sum(n), H, d) * spread).bfloat16() for n in (lq, lk, lq))
    k = (normal(g, sum(lk), H, d) * spread + normal(g, H, d)).bfloat16()
    cu_q, cu_k = (torch.tensor(R.offsets(n), dtype=torch.int32, device="cuda") for n in (lq, lk))
    o, lse = ts.ts_attn_fwd_kvcache(q, k, v, cu_q, cu_k, max(lq), max(lk), scale=scale, return_lse=True)
    return d_o, q, k, v, o, lse, cu_q, cu_k, max(lq), max(lk)


def check_attn(lq, lk, H, d, scale, got, args):
    ref, tol = R.packed_attn_bwd(*(x.double() for x in args[:6]), R.offsets(lq), R.offsets(lk), scale)
    for name, x, y, t in zip(("dq", "dk", "dv"), got, ref, tol):
        near(name, x, y, t)


ATTN = [  # query lengths, key lengths, heads, width
    ([1], [2], 1, 64),
    ([1], [1], 2, 128),
    ([2, 3], [5, 1], 3, 128),
    ([32], [32], 2, 128),
    ([64], [64], 2, 64),
    ([33], [65], 2, 64),
    ([256], [256], 1, 128),
    ([257], [129], 2, 128),
    ([1], [1000], 4, 64),
    ([1000], [1], 4, 128),
    ([300], [700], 3, 64),
    ([513], [777], 2, 128),
    ([0, 100, 0, 37, 1], [50, 0, 0, 300, 1], 2, 64),
    ([0, 100, 0, 37, 1], [50, 0, 0, 300, 1], 2, 128),
    ([777, 1, 0, 131, 600, 64], [777, 333, 100, 0, 900, 1], 3, 64),
    ([1300], [1300], 5, 128),
    ([17] * 70, [23] * 70, 2, 128),
    ([5] * 200, [9] * 200, 1, 64),
]


@pytest.mark.parametrize("splits", [1, 0, 3])
@pytest.mark.parametrize("case", ATTN, ids=lambda c: "%s-%s-%d-%d" % (c[0][:6], c[1][:6], c[2], c[3]))
def test_attn_bwd(case, splits):
    lq, lk, H, d = case
    say("attn_bwd", case, splits)
    scale = ts.default_scale(d)
    args = attn_inputs(lq, lk, H, d, scale, seed=4)
    got = ts.ts_attn_bwd(*args, num_splits=splits)
    check_attn(lq, lk, H, d, scale, got, args)
    again = ts.ts_attn_bwd(*args, num_splits=splits)
    assert all(same_bits(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0, 2.0 ** -100, 0.01])
def test_attn_bwd_scales(scale, d):
    say("scale", scale, d)
    lq, lk = [100, 40], [90, 200]
    args = attn_inputs(lq, lk, 2, d, scale, seed=5)
    got = ts.ts_attn_bwd(*args, scale=scale)
    check_attn(lq, lk, 2, d, scale, got, args)
