"""Angles of a base or a scaling that leads beyond the finite numbers are refused, and nothing is written."""
import ctypes as C
import math

import pytest

import paper_2412_01380_amd as D


@pytest.mark.parametrize("how", [
    dict(dims=4, base=1e4, kind=D.DIP_SCALING_BASE, factor=1e200), dict(dims=4, base=1e-4, kind=D.DIP_SCALING_BASE, factor=1e-200),
    dict(dims=64, base=1e4, kind=D.DIP_SCALING_LINEAR, factor=1e-310), dict(dims=64, base=1e-300, kind=D.DIP_SCALING_LINEAR, factor=1e-30),
    dict(dims=4, base=1e4, kind=D.DIP_SCALING_LIST, factors=[1.0, 1e-320]),
    dict(dims=8, base=1e4, kind=D.DIP_SCALING_PARTS, factor=1e-310, slow=1.0, fast=32.0, original_len=4096.0)])
def test_angles_beyond_the_finite_numbers(how):
    with pytest.raises(D.DipError, match="finite"):
        D.dip_rotary_frequencies(**how)
    out = (C.c_double * 2)(7.0, 7.0)
    scaling = D.libdip._RotaryScaling(D.DIP_SCALING_BASE, 0, 1e200, 0.0, 1.0, 1.0, None)
    assert D.lib.dip_rotary_frequencies(4, 1e4, C.byref(scaling), out) == D.DIP_ERR_INVALID_ARG
    assert list(out) == [7.0, 7.0]


def test_the_farthest_that_fit():
    f = D.dip_rotary_frequencies(4, 1e4, D.DIP_SCALING_BASE, factor=1e150)
    assert f[0] == 1.0 and abs(f[1] * 1e152 - 1) < 1e-12
    f = D.dip_rotary_frequencies(4, 1e-300, D.DIP_SCALING_LINEAR, factor=1e-100)
    assert math.isclose(f[1], 1e250, rel_tol=1e-12)
