"""Norm and rotation with one weight of the two on the GPU, and their gradients: the other rows are only turned."""
import pytest
import torch

import block_ref as R
from test_gpu_block import AXES, near, rope_inputs, rng, normal, same_bits, say

pytestmark = pytest.mark.gpu

ts = pytest.importorskip("paper_2606_19271_amd")


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ts.load()
    ts.load_block()


@pytest.mark.parametrize("turn", [True, False])
@pytest.mark.parametrize("which", ["q", "k"])
@pytest.mark.parametrize("T,Hq,Hk,d,interleaved,fused", [(1, 3, 2, 128, True, False), (333, 12, 5, 64, False, True), (1000, 40, 8, 128, True, True),
                                                         (9000, 20, 20, 128, False, False)])
def test_one_weight(T, Hq, Hk, d, interleaved, fused, which, turn):
    say("one weight", T, Hq, Hk, d, interleaved, fused, which, turn)
    q, k, pos, rope, wq, wk = rope_inputs(T, Hq, Hk, d, True, turn, interleaved, fused, 1000, 75)
    wq, wk = (wq, None) if which == "q" else (None, wk)
    g = rng(76)
    dq, dk = normal(g, T, Hq, d).bfloat16(), normal(g, T, Hk, d).bfloat16()
    angle = R.angles(pos, rope.freq, AXES[d]) if turn else None
    got = ts.ts_qk_rope(q, k, pos, rope, wq, wk, eps=1e-6)
    # (what has no weight is not read back)
    back = ts.ts_qk_rope_bwd(dq, dk, q if wq is not None else None, k if wk is not None else None, pos, rope, wq, wk, eps=1e-6)
    for i, (x, dy, w) in enumerate(((q, dq, wq), (k, dk, wk))):
        w = None if w is None else w.double()
        ref, mag = (f(x.double(), w, angle, interleaved, 1e-6) for f in (R.rope, R.rope_slack))
        near("y", got[i], ref, R.HALF * ref.abs() + 1.01 * R.FINE * mag)
        dx, dw, mag, mag_w = R.rope_bwd(dy.double(), x.double(), w, angle, interleaved, 1e-6)
        near("dx", back[i], dx, R.HALF * dx.abs() + 1.01 * R.FINE * mag)
        if w is None:
            assert back[2 + i] is None
            if not turn:
                assert same_bits(got[i], x) and same_bits(back[i], dy)
        else:
            near("dw", back[2 + i], dw, R.FINE * mag_w)
