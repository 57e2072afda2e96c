"""The shapes of test_gpu_cross_shares.py are dealt out as that test needs them."""
import pytest

from paper_2509_01085_amd import binding as B

import cross_deal as D
from test_gpu_cross_shares import SHORT_UNITS


@pytest.mark.parametrize("name", list(SHORT_UNITS))
def test_units_of_two_tiles_follow_other_pieces_of_their_workgroup(name):
    s, lens = SHORT_UNITS[name]
    assert D.rows_deal(s)[0] and D.short_units_behind_others(s, lens) >= 40


@pytest.mark.parametrize("name", list(SHORT_UNITS))
def test_the_restated_deal_is_the_librarys(name):
    """A workgroup of a launch in shares has two places for partial results, of so many floats a lane for each of four wavefronts."""
    s, lens = SHORT_UNITS[name]
    shares, grid, tile, rows = D.rows_deal(s)
    values, left = divmod(B.cross_fwd_workspace_bytes(s), grid * 2 * 4 * 64 * 4)
    assert left == 0 and 0 <= values - (32 if s.d <= 64 else 64) < 8
    got = [p for w in D.pieces(s, lens) for p in w]
    assert sum(p[3] for p in got) == rows * sum(-(-min(n, s.S) // tile) for n in lens)
    assert B.cross_fwd_workspace_bytes(B.CrossShape(1, 12, 12, 33280, 512, 128, B.BF16)) == 0
