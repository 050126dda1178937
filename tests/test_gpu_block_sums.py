"""Long sums of the norm weights' gradients on the GPU."""
import pytest
import torch

import block_ref as R
from test_gpu_block import AXES, near, normal, rng, say

pytestmark = pytest.mark.gpu

ts = pytest.importorskip("paper_2606_19271_amd")


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ts.load()
    ts.load_block()


@pytest.mark.parametrize("T,Hq,Hk,d", [(1 << 22, 1, 1, 64), ((1 << 22) + 17, 1, 0, 128), (1 << 19, 33, 5, 64)])
def test_equal_terms_of_millions_of_tokens(T, Hq, Hk, d):
    """Every token has the same rows, so that every rounding of a running sum goes the same way: 32 bits lose half a step a term there,
    2^-25 of the sum times their number.  The bound is that of chains of 256."""
    say("equal terms", T, Hq, Hk, d)
    g = rng(70)
    wq, wk = 1 + 0.3 * normal(g, d), 1 + 0.3 * normal(g, d)
    r, pos = ts.rope(AXES[d]), torch.tensor([[3, 1, 4]], dtype=torch.int32, device="cuda").expand(T, 3).contiguous()
    rows = [(normal(g, 1, H, d) * 2).bfloat16() if H else None for H in (Hq, Hk, Hq, Hk)]  # queries, keys, and their results' gradients
    q, k, dq, dk = (None if x is None else x.expand(T, -1, -1).contiguous() for x in rows)
    got = ts.ts_qk_rope_bwd(dq, dk, q, k, pos, r, wq, wk if Hk else None)
    for i, w in ((0, wq), (1, wk)):
        if rows[i] is None:
            assert got[2 + i] is None
            continue
        dx, dw, mag, mag_w = R.rope_bwd(rows[2 + i].double(), rows[i].double(), w.double(), R.angles(pos[:1], r.freq, AXES[d]), True, 1e-6)
        near("dw", got[2 + i], T * dw, R.FINE * T * mag_w)
        near("dx", got[i][-1:], dx, R.HALF * dx.abs() + 1.01 * R.FINE * mag)


@pytest.mark.parametrize("d", [64, 128])
def test_chains_that_end_anywhere(d):
    """Sizes whose waves take a step or two fewer or more than a chain's, or as many."""
    for T in (128 * 2048, 128 * 2048 - 1, 128 * 2048 + 1, 127 * 2048 + 3, 257 * 2048):
        say("chain", T, d)
        g = rng(71)
        x, dy = normal(g, T, 1, d).bfloat16(), normal(g, T, 1, d).bfloat16()
        w = 1 + 0.3 * normal(g, d)
        dx, _, dw, _ = ts.ts_qk_rope_bwd(dy, None, x, None, q_weight=w)
        want, want_w, mag, mag_w = R.rope_bwd(dy.double(), x.double(), w.double(), None, True, 1e-6)
        near("dx", dx, want, R.HALF * want.abs() + 1.01 * R.FINE * mag)
        near("dw", dw, want_w, R.FINE * mag_w)
