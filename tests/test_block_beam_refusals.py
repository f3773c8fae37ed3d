"""Calls of block products and of decoding by beams that would race or leave the arrays: refused before anything is enqueued.  No compute
call is made here."""
import ctypes as C

import pytest

from .test_score_args import PTR, _struct


@pytest.fixture(scope="module")
def B():
    from paper_2605_28396_amd import binding
    return binding


def test_words_of_excluded_rows_are_not_those_written(B):
    base = dict(N=50, ld_x=64, H=64, x_dtype=0, f8=0, tile=1, x=PTR, q=PTR, scale=PTR, row_status=PTR + 4096)
    for at in (0, 4, -4, 196, -196):
        p = _struct(B.adwin_opd_block_rows_problem, base, dict(x_status=PTR + 4096 + at))
        assert B.lib.adwin_opd_block_rows(C.byref(p), None) == B.ADWIN_E_ALIGN, at
    p = _struct(B.adwin_opd_block_rows_problem, base, dict(N=0, x_status=PTR + 4096))
    assert B.lib.adwin_opd_block_rows(C.byref(p), None) == B.ADWIN_OK
