"""The operators around the attention refuse workspaces and tables at addresses that their kernels' accesses do not fit."""
import ctypes as C

import pytest

from paper_2509_01085_amd import binding as B

from test_operators_host import CROSS, ROPE, SHAPE, bwd, cbwd, cfwd, fwd, p


@pytest.mark.parametrize("off", (1, 4, 8))
def test_workspaces_are_16_byte_aligned(off):
    few = B.CrossShape(1, 1, 1, 1, 100000, 128, B.BF16)  # its keys are split: the forward needs scratch
    assert cfwd(few, ws=p + off) == -9 and cbwd(few, ws=p + off) == -9 and cbwd(CROSS, ws=p + off) == -9
    assert bwd(ws=p + off) == -9
    assert cfwd(few, ws=None) == -7 and cbwd(ws=None) == -7 and bwd(ws=None) == -7  # as before


def test_a_rotation_table_is_8_byte_aligned():
    table = lambda t: B.lib().bsa_rope_table(C.byref(SHAPE.c()), C.byref(ROPE.c()), 1e4, 0, 0, 0, t, None)  # noqa: E731
    for t in (p + 1, p + 4):
        assert fwd(table=t) == -9 and bwd(table=t) == -9 and table(t) == -9
    for rope in (None, B.Rope(0, 0, 0)):  # one that is not read may lie anywhere: the next check is what refuses
        assert fwd(table=p + 4, rope=rope, xs=None) == -1 and bwd(table=p + 4, rope=rope, dxs=None) == -1
