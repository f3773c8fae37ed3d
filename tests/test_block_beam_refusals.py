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


def _reorder(B, n, K, **state):
    """The status of a move of `n` sequences of K beams, one array at PTR to 2^45 bytes behind it."""
    s = (B.adwin_opd_beam_state * 1)()
    for k, v in {**{"from": PTR, "to": PTR + (1 << 45), "positions": 16, "bytes": 4, "planes": 1}, **state}.items():
        setattr(s[0], k, v)
    p = B.adwin_opd_beam_reorder_problem(C.sizeof(B.adwin_opd_beam_reorder_problem), n, K, K, 1, 0, C.addressof(s), PTR - 64, None)
    return B.lib.adwin_opd_beam_reorder(C.byref(p), None)


def test_moves_of_rows_beyond_any_address_are_refused(B):
    """Distances of rows whose sum leaves 64 bits: such planes and rows count as apart, and such arrays as without end, if it is not looked at."""
    far, n = (1 << 40) - 16, (1 << 18) - 1                           # 2^24 - 64 rows: (rows - 1) far is 2^64 and little less
    assert _reorder(B, n, 64, from_row=far, to_row=far) == B.ADWIN_E_SHAPE
    assert _reorder(B, n, 64, from_row=64, to_row=far) == _reorder(B, n, 64, from_row=far, to_row=64) == B.ADWIN_E_SHAPE
    # the rows of one plane lie over the other planes
    assert _reorder(B, n, 64, from_row=far, to_row=far, planes=10, from_plane=1 << 39, to_plane=1 << 39) == B.ADWIN_E_SHAPE
    assert _reorder(B, 1 << 17, 64, from_row=far, to_row=far) == B.ADWIN_E_SHAPE              # 2^63 and little less
    planes = (1 << 20) - 1
    assert _reorder(B, 1, 1, planes=planes, from_plane=far, to_plane=far) == B.ADWIN_E_SHAPE
    # 2^48 bytes from the first to the last, and 16 fewer: only these get as far as a move in place that is none
    edge = dict(to=PTR, planes=257, from_plane=far, to_plane=far - 16)
    assert _reorder(B, 1, 1, positions=1024, **edge) == B.ADWIN_E_SHAPE and _reorder(B, 1, 1, positions=1020, **edge) == B.ADWIN_E_ALIGN


def test_selections_over_what_they_read_are_refused(B):
    """Other sequences may still be read: only with keep = K do new scores, ends and lengths go where the old ones are, exactly."""
    names = ("z", "score", "finished", "length", "parent", "token", "new_score", "new_finished", "new_length", "row_status")
    at = {n: PTR + (i + 1) * (1 << 20) for i, n in enumerate(names)}
    base = dict(B=7, ld_z=1000, K=3, keep=3, V=1000, z_dtype=0, end=-1, temperature=1.0, length_power=0.0, **at)
    ws = PTR + (1 << 30)

    def st(workspace=ws, **over):
        p = _struct(B.adwin_opd_beam_select_problem, base, over)
        return B.lib.adwin_opd_beam_select(C.byref(p), workspace, 1 << 28, None)
    need = B.adwin_opd_beam_select_workspace_bytes(_struct(B.adwin_opd_beam_select_problem, base, {}))
    read, written = names[:4], names[4:]
    old = {"new_" + n: n for n in ("score", "finished", "length")}
    for w in written:
        for r in names:
            if r == w:
                continue
            for keep, offset in ((2, 0), (3, 4), (3, -4), (3, 0), (4, 0), (4, 80), (4, -108)):     # 84 bytes of beams, 112 of four kept
                if (keep == 3 and offset == 0 and old.get(w) == r) or (keep == 4 and offset == -108 and w == "row_status"):
                    continue
                assert st(keep=keep, **{w: at[r] + offset}) == B.ADWIN_E_ALIGN, (w, r, keep, offset)
    assert st(parent=at["z"] + 2 * (20 * 1000 + 1000) - 4) == B.ADWIN_E_ALIGN                      # the last logits
    for name in names:
        assert st(**{name: ws + need - 4}) == B.ADWIN_E_ALIGN, name
    # the old ones' places, but another is in the way
    assert st(new_score=at["score"], new_length=at["score"]) == st(new_score=at["finished"]) == B.ADWIN_E_ALIGN
