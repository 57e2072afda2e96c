"""The norm's eps is a normal float: the kernels' reciprocal square root takes smaller ones for zero, and rows of zeros would be NaN."""
import pytest

from test_operators_host import bwd, fwd

TINY = 2.0 ** -126


@pytest.mark.parametrize("eps", (TINY * (1 - 2.0 ** -23), 1e-38, 1e-40, 2.0 ** -149))
def test_a_subnormal_eps_is_refused(eps):
    assert fwd(eps=eps, xs=None) == -3 and bwd(eps=eps, dxs=None) == -3


def test_the_least_normal_one_is_taken():
    assert fwd(eps=TINY, xs=None) == -1 and bwd(eps=TINY, dxs=None) == -1  # the next check refuses
