"""Attention's gradients on the GPU within the sharper bounds of tests/block_bounds.py."""
import math

import pytest
import torch

import block_bounds as B
import block_ref as R
from test_gpu_block import ATTN, attn_inputs, normal, rng, say

pytestmark = pytest.mark.gpu

ts = pytest.importorskip("paper_2606_19271_amd")


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ts.load()
    ts.load_block()


def bounded(lq, lk, args, scale, splits):
    """ts_attn_bwd of these arguments: every gradient within its bounds.  Returns dq and its definition."""
    got = ts.ts_attn_bwd(*args, scale=scale, num_splits=splits)
    want = B.packed(*(x.double() for x in args[:6]), R.offsets(lq), R.offsets(lk), scale)
    for name, x, (ref, tol, most) in zip(("dq", "dk", "dv"), got, want):
        B.check(name, x, ref, tol, most, say)
    return got[0], want[0][0]


def within(lq, lk, d, q, k, v, d_o, splits):
    """The same with the result and the log-sum-exp of the definition."""
    scale = ts.default_scale(d)
    cu_q, cu_k = (torch.tensor(R.offsets(n), dtype=torch.int32, device="cuda") for n in (lq, lk))
    o, lse = R.packed_attn(*(x.double() for x in (q, k, v)), R.offsets(lq), R.offsets(lk), scale)
    return bounded(lq, lk, (d_o, q, k, v, o.bfloat16(), lse.float(), cu_q, cu_k, max(lq), max(lk)), scale, splits)


@pytest.mark.parametrize("splits", [1, 0, 3])
@pytest.mark.parametrize("case", ATTN, ids=lambda c: "%s-%s-%d-%d" % (c[0][:6], c[1][:6], c[2], c[3]))
def test_gradients_within_their_bounds(case, splits):
    lq, lk, H, d = case
    say("bounds", case, splits)
    scale = ts.default_scale(d)
    bounded(lq, lk, attn_inputs(lq, lk, H, d, scale, seed=63), scale, splits)


@pytest.mark.parametrize("splits", [1, 0, 5])
@pytest.mark.parametrize("mean", [1, 4, 8])
@pytest.mark.parametrize("lq,lk,H,d", [([300, 500], [1000, 700], 3, 64), ([300, 500], [1000, 700], 3, 128), ([2900, 300], [2048, 2500], 12, 128)])
def test_keys_with_a_mean(lq, lk, H, d, mean, splits):
    """In small tiles and in large ones: what the keys have in common does not go into dq's error."""
    say("mean", lq, lk, H, d, mean, splits)
    g = rng(64)
    q, v, d_o = (normal(g, sum(n), H, d) for n in (lq, lk, lq))
    k = normal(g, sum(lk), H, d) + mean * normal(g, H, d).sign()
    within(lq, lk, d, (0.3 * q).bfloat16(), k.bfloat16(), v.bfloat16(), d_o.bfloat16(), splits)


@pytest.mark.parametrize("splits", [1, 0, 3])
@pytest.mark.parametrize("shift", [2, 8, 64])
@pytest.mark.parametrize("d", [64, 128])
def test_first_keys_that_stand_apart(d, shift, splits):
    """The first 32 keys of a segment lie far from the others in every channel and have next to no weight: dq is off by its own
    rounding whatever they are."""
    say("first keys", d, shift, splits)
    lq, lk, H = [256, 100], [3120, 700], 2
    g = rng(60)
    q, v, d_o = normal(g, sum(lq), H, d), normal(g, sum(lk), H, d).bfloat16(), normal(g, sum(lq), H, d).bfloat16()
    k, u = normal(g, sum(lk), H, d), normal(g, H, d).sign()
    for at in (0, lk[0]):
        k[at:at + 32] += shift * u
    q = 0.3 * q
    q = q - (q * u).sum(-1, keepdim=True) * u / d - 1.2 / math.sqrt(d) * u  # (their scores are -1.2 times the shift)
    dq, ref = within(lq, lk, d, q.bfloat16(), k.bfloat16(), v, d_o, splits)
    # 0.0017 of its norm, HALF / sqrt(3) = 0.00226 where every element is at the low end of its binade
    assert (dq.double() - ref).norm() < 0.0020 * ref.norm()


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("share", [0.01, 0.7, 1.0])
@pytest.mark.parametrize("d", [64, 128])
def test_keys_that_one_channel_masks(d, share, splits):
    """A channel that is 1 in every query and -30000 in the keys that are to have no weight (1.0: in all but one)."""
    say("masking channel", d, share, splits)
    lq, lk, H = [130, 70], [1000, 333], 2
    g = rng(61)
    q, k, v, d_o = (normal(g, sum(n), H, d).bfloat16() for n in (lq, lk, lk, lq))
    q[..., 3] = 1
    hidden = torch.rand(sum(lk), generator=g, device="cuda") < share
    hidden[[7, 1200]] = False
    k[hidden, :, 3] = -30000
    dq, ref = within(lq, lk, d, q, k, v, d_o, splits)
    if share < 1:
        # its own rounding, HALF / sqrt(3) of its norm at most; 400 elements, four deviations
        assert (dq[..., 3].double() - ref[..., 3]).norm() < R.HALF * math.sqrt((1 + 4 * math.sqrt(2 / 400)) / 3) * ref[..., 3].norm()


@pytest.mark.parametrize("H", [1, 2])
@pytest.mark.parametrize("d", [64, 128])
def test_three_keys_of_weight_anywhere(d, H):
    """64 segments in which all keys but three are 30000 in one channel, and have no weight by it; the three lie at another place of a
    64-key tile in each segment, and the channel is another one."""
    say("every key", d, H)
    n, lq, lk = 195, [5] * 64, [195] * 64
    g = rng(62)
    q, k, v, d_o = (normal(g, sum(x), H, d).bfloat16() for x in (lq, lk, lk, lq))
    for s in range(64):
        c, hidden = 37 * s % d, torch.ones(n, dtype=torch.bool, device="cuda")
        hidden[[s, s + 64, s + 128]] = False
        q[5 * s:5 * s + 5, :, c] = -1
        k[n * s:n * s + n, :, c].masked_fill_(hidden[:, None], 30000)
    for splits in (1, 0):
        within(lq, lk, d, q, k, v, d_o, splits)
