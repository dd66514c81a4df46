"""Sizes of a norm's and a rotation's numbers that are refused, and the last ones that
aren't, on the CPU."""
import ctypes
import math

import pytest

from paper_2607_03333_amd import spork
from test_rows_abi_host import INVAL, norm, rope, turn, write


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


@pytest.mark.parametrize("call", (turn, write))
def test_magnitudes_that_32_bits_hold(call):
    """Cosines and sines are multiplied by the magnitude and kept in 32 bits: past them they would be infinities, below
    them lose their places."""
    for m in (3.5e38, -3.5e38, 1e300, -math.inf, math.nan, 1.1e-38, -1e-45, 5e-324):
        assert b"magnitude" in why(call, rope=rope(magnitude=m)), m
    for m in (0.0, 1.0, -0.5, 3.4e38, -3.4e38, 1.2e-38, -1.2e-38):
        assert b"positions" in why(call, rope=rope(magnitude=m)), m


def test_frequencies_that_are_no_numbers():
    """Factors under which a frequency passes 2^1024 are refused, and nothing is written."""
    call, f, m = spork.lib().spork_rope_frequencies, (ctypes.c_double * 64)(*[7.0] * 64), ctypes.c_double(7)
    for kind, factor in ((spork.SPORK_ROPE_SCALE_LINEAR, 5e-324), (spork.SPORK_ROPE_SCALE_BASE, 5e-324),
                         (spork.SPORK_ROPE_SCALE_PARTS, 1e-310), (spork.SPORK_ROPE_SCALE_BANDS, 1e-310)):
        s = spork.spork_rope_scaling(kind, 4096, factor, 32.0, 1.0)
        assert call(128, 1e4, ctypes.byref(s), f, ctypes.byref(m)) == INVAL, kind
        assert b"factor" in spork.lib().spork_last_error() and m.value == 7 and list(f) == [7.0] * 64
    s = spork.spork_rope_scaling(spork.SPORK_ROPE_SCALE_LINEAR, 0, 1e-300, 0.0, 0.0)
    assert call(128, 1e4, ctypes.byref(s), f, ctypes.byref(m)) == 0 and all(map(math.isfinite, f)) and m.value == 1
