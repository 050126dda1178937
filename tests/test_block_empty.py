"""Attention's gradients of no segments (no GPU): nothing is done, and in validation mode rows that belong to none are named."""
import pytest

from test_block_abi import bwd, refused

pytest.importorskip("paper_2606_19271_amd")
from paper_2606_19271_amd import _lib  # noqa: E402
from paper_2606_19271_amd import block as B  # noqa: E402


def test_rows_of_no_segment(monkeypatch):
    lib = B.load_block()
    rows = ({}, {"Tq": 0}, {"Tk": 0})
    for x in rows:
        assert bwd(lib, nseq=0, **x) == _lib.TS_OK
    monkeypatch.setenv("TS_ATTN_VALIDATE", "1")
    for x in rows:
        refused(bwd(lib, nseq=0, **x), "TS_ERR_SEGMENTS")
    assert bwd(lib, nseq=0, Tq=0, Tk=0) == _lib.TS_OK
