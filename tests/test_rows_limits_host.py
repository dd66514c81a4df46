"""Sizes of a norm's and a rotation's numbers that are refused, and the last ones that
aren't, on the CPU."""
import math

import pytest

from paper_2607_03333_amd import spork
from test_rows_abi_host import INVAL, norm, turn, write


def why(call, **kw):
    """What a call that is refused anyway, for its positions if for nothing in front of them, is refused for."""
    assert call(positions=None, **kw) == INVAL
    return spork.lib().spork_last_error()


@pytest.mark.parametrize("call", (turn, write))
def test_eps_up_to_2_100(call):
    for eps in (math.nextafter(2.0 ** 100, math.inf), 1e39, 1e300, math.inf, math.nan, -5e-324):
        assert b"eps" in why(call, norm=norm(eps=eps)), eps
    for eps in (0.0, 5e-324, 1e-6, 2.0 ** 100):
        assert b"positions" in why(call, norm=norm(eps=eps)), eps
