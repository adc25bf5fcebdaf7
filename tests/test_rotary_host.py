"""Host-side checks of the calls that turn rows to their positions: angles against their formulas, bad arguments refused
before the HIP runtime is touched, and the oracle on cases worked by hand."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import decode_oracle as O
from test_decode_host import BAD_BATCHES, BAD_CACHES, FAKE, batch, cache


@pytest.fixture(scope="module")
def D():
    import paper_2412_01380_amd as D
    return D


def rotary(**over):
    from paper_2412_01380_amd.libdip import _Rotary
    f = dict(freq=FAKE, dims=128, layout=0, scale=1.0, reserved=0)
    f.update(over)
    return _Rotary(*[f[n] for n, _ in _Rotary._fields_])


@pytest.mark.parametrize("dims", [2, 6, 64, 128])
def test_angles(D, dims):
    i = np.arange(dims // 2)
    f = 10000.0 ** (-2 * i / dims)
    close = lambda a, b: np.allclose(np.asarray(a), b, rtol=1e-14, atol=0)
    assert close(D.dip_rotary_frequencies(dims), f)
    assert close(D.dip_rotary_frequencies(dims, 500000.0), 500000.0 ** (-2 * i / dims))
    assert close(D.dip_rotary_frequencies(dims, kind=D.DIP_SCALING_LINEAR, factor=4.0), f / 4)
    if dims > 2:
        g = D.dip_rotary_frequencies(dims, kind=D.DIP_SCALING_BASE, factor=8.0)
        assert close(g, (10000.0 * 8 ** (dims / (dims - 2))) ** (-2 * i / dims))
        assert math.isclose(g[0], 1.0) and math.isclose(g[-1], f[-1] / 8, rel_tol=1e-12)    # the slowest pair by all of it
    each = 1 + 0.1 * i
    assert close(D.dip_rotary_frequencies(dims, kind=D.DIP_SCALING_LIST, factors=list(each)), f / each)
    turns = 4096 * f / (2 * math.pi)
    m = np.clip((turns - 1) / (32 - 1), 0, 1)
    assert close(D.dip_rotary_frequencies(dims, kind=D.DIP_SCALING_PARTS, factor=8.0, slow=1, fast=32, original_len=4096), f * m + f / 8 * (1 - m))


def test_angles_are_refused(D):
    bad = [dict(dims=0), dict(dims=3), dict(base=0.0), dict(base=math.nan), dict(base=math.inf), dict(kind=5), dict(kind=-1),
           dict(kind=1, factor=0.0), dict(kind=1, factor=math.nan), dict(kind=2, factor=2.0, dims=2), dict(kind=3, factor=2.0),
           dict(kind=3, factor=2.0, original_len=10.0, slow=2.0, fast=2.0), dict(kind=3, factor=2.0, original_len=10.0, slow=-1.0),
           dict(kind=3, factor=2.0, original_len=10.0, slow=math.nan), dict(kind=4), dict(kind=4, factors=[1.0, 0.0]),
           dict(kind=4, factors=[1.0, math.inf])]
    for over in bad:
        a = dict(dims=4, base=10000.0)
        a.update(over)
        with pytest.raises(D.DipError) as e:
            D.dip_rotary_frequencies(**a)
        assert e.value.status == D.DIP_ERR_INVALID_ARG, over
    with pytest.raises(TypeError):
        D.dip_rotary_frequencies(8, kind=4, factors=[1.0])
    assert D.lib.dip_rotary_frequencies(4, 1.0, None, None) == D.DIP_ERR_INVALID_ARG


BAD_ROTARY = [
    (dict(freq=None), "INVALID_ARG"), (dict(reserved=1), "INVALID_ARG"), (dict(layout=2), "INVALID_ARG"), (dict(layout=-1), "INVALID_ARG"),
    (dict(dims=0), "INVALID_ARG"), (dict(dims=63), "INVALID_ARG"), (dict(dims=130), "INVALID_ARG"), (dict(scale=math.nan), "INVALID_ARG"),
    (dict(scale=math.inf), "INVALID_ARG"), (dict(freq=FAKE + 4), "UNSUPPORTED"),
]


def append(D, c=None, b=None, r=None, layer=0, parents=None, q=FAKE, qs=512, heads=4, out=0x20000, os=512, k=0x30000, v=0x40000, rs=256):
    c, b, r = c or cache(), b or batch(), r or rotary()
    return D.lib.dip_kv_append_rotary(C.byref(c), layer, C.byref(b), parents, C.byref(r), q, qs, heads, out, os, k, v, rs, None)


def rotate(D, r=None, x=FAKE, xs=512, pos=FAKE, rows=3, heads=4, dims=128, dtype=1, out=0x20000, os=512):
    r = r or rotary()
    return D.lib.dip_rotate_rows(C.byref(r), x, xs, pos, rows, heads, dims, dtype, out, os, None)


@pytest.mark.parametrize("over,status", BAD_ROTARY)
def test_descriptors_are_refused(D, over, status):
    want = getattr(D, "DIP_ERR_" + status)
    assert append(D, r=rotary(**over)) == want
    assert rotate(D, r=rotary(**over)) == want
    assert "rotary" in D.dip_last_error()


@pytest.mark.parametrize("over,status", BAD_CACHES)
def test_caches_are_refused(D, over, status):
    assert append(D, c=cache(**over), r=rotary(dims=8)) == getattr(D, "DIP_ERR_" + status)


@pytest.mark.parametrize("over,status", BAD_BATCHES)
def test_batches_are_refused(D, over, status):
    assert append(D, b=batch(**over)) == getattr(D, "DIP_ERR_" + status)


def test_append_arguments_are_refused(D):
    I, U = D.DIP_ERR_INVALID_ARG, D.DIP_ERR_UNSUPPORTED
    assert append(D, layer=2) == I and append(D, layer=-1) == I
    assert append(D, k=None) == I and append(D, v=None) == I
    assert append(D, q=None) == I and append(D, out=None) == I and append(D, heads=0) == I and append(D, heads=-1) == I
    assert append(D, qs=504) == I and append(D, os=504) == I and append(D, rs=248) == I
    assert append(D, qs=516) == U and append(D, os=516) == U and append(D, rs=260) == U
    assert append(D, q=FAKE + 2) == U and append(D, k=0x30008) == U and append(D, v=0x40004) == U and append(D, out=0x20008) == U
    assert append(D, heads=65536, qs=1 << 24, os=1 << 24) == U
    assert append(D, parents=FAKE, b=batch(n_rows=100, max_rows=65)) == U
    # 5 rows of 512 elements of 2 bytes: what overlaps
    assert append(D, out=FAKE + 512) == I and "overlap" in D.dip_last_error()
    assert append(D, out=FAKE + 1024) == I
    assert append(D, out=0x30000 - 16) == I and append(D, out=0x40000) == I
    assert append(D, out=FAKE, os=520) == I                                     # q itself with another stride
    assert append(D, qs=1024, os=1024, out=FAKE + 512) == I                     # columns of one array that meet


def test_rotate_arguments_are_refused(D):
    I, U = D.DIP_ERR_INVALID_ARG, D.DIP_ERR_UNSUPPORTED
    assert rotate(D, x=None) == I and rotate(D, pos=None) == I and rotate(D, out=None) == I
    assert rotate(D, dtype=2) == U
    assert rotate(D, rows=0) == I and rotate(D, heads=0) == I and rotate(D, dims=0) == I
    assert rotate(D, rows=1 << 24) == U and rotate(D, heads=65536) == U and rotate(D, dims=65544) == U
    assert rotate(D, r=rotary(dims=8), dims=12) == U and rotate(D, r=rotary(dims=2), dims=6, dtype=0) == U
    assert rotate(D, xs=504) == I and rotate(D, os=504) == I and rotate(D, xs=516) == U and rotate(D, os=516) == U
    assert rotate(D, x=FAKE + 2) == U and rotate(D, out=0x20008) == U
    assert rotate(D, out=FAKE + 1024) == I and rotate(D, out=FAKE, os=520) == I
    assert rotate(D, r=rotary(dims=4098), dims=8192, xs=1 << 20, os=1 << 20) == U


def test_oracle_turns_by_hand():
    x = np.array([[[1.0, 0.0, 5.0, 0.0, 2.0, 7.0]]])
    half = O.turn(x, [1], [math.pi / 2, math.pi], False)           # pairs (0, 2), (1, 3); 4, 5 pass through
    assert np.allclose(half, [[[-5, 0, 1, 0, 2, 7]]])
    inter = O.turn(x, [-1], [math.pi / 2, math.pi], True, 2.0)     # pairs (0, 1), (2, 3)
    assert np.allclose(inter, [[[0, -2, -10, 0, 2, 7]]])
    assert O.tree_positions(7, [-1, 0, 0, 2, 9, 4]) == [7, 8, 8, 9, 7, 7]
