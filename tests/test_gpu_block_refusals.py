"""What the binding of the block's calls refuses of tensors on the GPU."""
import pytest
import torch

pytestmark = pytest.mark.gpu

ts = pytest.importorskip("paper_2606_19271_amd")


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ts.load()
    ts.load_block()


def test_rows_of_no_segment():
    """Offsets of one entry have no segment: gradients of rows would be left as the allocator made them."""
    x, none = (torch.ones(n, 2, 64, dtype=torch.bfloat16, device="cuda") for n in (5, 0))
    lse, cu = torch.zeros(5, 2, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    for q, k, s in ((x, x, lse), (none, x, lse[:0]), (x, none, lse)):
        with pytest.raises(ValueError):
            ts.ts_attn_bwd(q, q, k, k, q, s, cu, cu, 5, 5)
    dq, dk, dv = ts.ts_attn_bwd(none, none, none, none, none, lse[:0], cu, cu, 5, 5)
    assert dq.shape == dk.shape == dv.shape == none.shape
