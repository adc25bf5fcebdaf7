"""Host-side checks of the calls over blocks of a long context: bad arguments are refused before the HIP runtime is
touched, sizes, and the oracle on cases worked by hand."""
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


def bounds(D, c=None, layer=0, n_layers=1, seqs=FAKE, n=2, back=5, block=16, to=FAKE):
    c = c or cache()
    return D.lib.dip_kv_block_bounds(C.byref(c), layer, n_layers, seqs, n, back, block, to, None)


def select(D, c=None, b=None, layer=0, q=FAKE, qs=512, heads=4, block=16, bo=FAKE, n=3, sinks=1, recent=8, out=FAKE, ws=FAKE, size=1 << 40):
    c, b = c or cache(), b or batch()
    return D.lib.dip_select_blocks(C.byref(c), layer, C.byref(b), q, qs, heads, block, bo, n, sinks, recent, out, ws, size, None)


def attend(D, c=None, b=None, layer=0, parents=None, bl=FAKE, n=3, block=16, q=FAKE, qs=512, heads=4, scale=0.1, sinks=1, recent=8, out=FAKE,
           os=512, ws=FAKE, size=1 << 40):
    c, b = c or cache(), b or batch()
    return D.lib.dip_block_attention(C.byref(c), layer, C.byref(b), parents, bl, n, block, q, qs, heads, scale, sinks, recent, out, os, ws, size, None)


@pytest.mark.parametrize("over,status", BAD_CACHES)
def test_caches_are_refused(D, over, status):
    want, c, b = getattr(D, "DIP_ERR_" + status), cache(**over), batch()
    assert bounds(D, c) == want and select(D, c) == want and attend(D, c) == want
    assert D.lib.dip_block_bounds_bytes(C.byref(c), 16) == 0
    assert D.lib.dip_select_blocks_workspace_bytes(C.byref(c), C.byref(b), 4, 16) == 0
    assert D.lib.dip_block_attention_workspace_bytes(C.byref(c), C.byref(b), 4, 16, 3, 1, 8) == 0


@pytest.mark.parametrize("over,status", BAD_BATCHES)
def test_batches_are_refused(D, over, status):
    want = getattr(D, "DIP_ERR_" + status)
    assert select(D, b=batch(**over)) == want and attend(D, b=batch(**over)) == want


def test_arguments_are_refused(D):
    I, U, W = D.DIP_ERR_INVALID_ARG, D.DIP_ERR_UNSUPPORTED, D.DIP_ERR_WORKSPACE
    for block in (0, 8, 24, 32, -16):                                # (pages of 16 slots)
        assert bounds(D, block=block) == U and select(D, block=block) == U and attend(D, block=block) == U
    assert bounds(D, layer=2) == I and bounds(D, layer=1, n_layers=2) == I and bounds(D, n_layers=0) == I and bounds(D, layer=-1) == I
    assert bounds(D, seqs=None) == I and bounds(D, to=None) == I and bounds(D, n=0) == I and bounds(D, n=65536) == I
    assert bounds(D, back=-1) == I and bounds(D, to=FAKE + 8) == U
    for call in (select, attend):
        assert call(D, c=cache(head_dim=80, slot_stride=80)) == U
        assert call(D, layer=2) == I and call(D, layer=-1) == I
        assert call(D, q=None) == I and call(D, qs=504) == I and call(D, qs=516) == U and call(D, q=FAKE + 8) == U
        assert call(D, heads=3) == I and call(D, heads=0) == I and call(D, heads=65536, qs=1 << 24) == U
        assert call(D, n=0) == I and call(D, n=D.DIP_MAX_SELECT + 1) == U
        assert call(D, sinks=-1) == I and call(D, recent=-1) == I
        assert call(D, ws=None) == W and call(D, ws=FAKE + 16) == W and call(D, size=16) == W
    assert select(D, bo=None) == I and select(D, out=None) == I and select(D, bo=FAKE + 8) == U
    assert attend(D, bl=None) == I and attend(D, out=None) == I
    assert attend(D, os=504) == I and attend(D, os=516) == U and attend(D, out=FAKE + 8) == U
    assert attend(D, parents=FAKE, b=batch(n_rows=100, max_rows=65)) == U
    for scale in (0.0, -1.0, math.nan, math.inf):
        assert attend(D, scale=scale) == I


def test_sizes(D):
    c, b = cache(page_size=64, page_stride=64 * 256, head_stride=64 * 128), batch()
    assert D.lib.dip_block_bounds_bytes(C.byref(c), 16) == 2 * 9 * 2 * 4 * 2 * 128 * 2
    for rows in (1, 64, 5000):
        b = batch(n_rows=rows, max_rows=rows)
        assert D.lib.dip_select_blocks_workspace_bytes(C.byref(c), C.byref(b), 8, 32) >= rows * 2 * 8 * 4
        for n in (1, 64, 4096):
            assert 256 <= D.lib.dip_block_attention_workspace_bytes(C.byref(c), C.byref(b), 8, 32, n, 4, 0x7fffffff) <= 64 << 20
    # a launch has fewer than 2^32 threads
    many = cache(n_kv_heads=512, page_stride=16 * 512 * 128)
    assert attend(D, c=many, b=batch(n_rows=1 << 18, max_rows=1 << 18), heads=512, qs=65536, os=65536) == D.DIP_ERR_UNSUPPORTED
    assert "too many rows" in D.dip_last_error()


def test_oracle_by_hand():
    assert O.block_parts(100, 16, 16, 3, 20) == (16, 80) and O.block_parts(100, 16, 16, 3, 0) == (16, 96)
    assert O.block_parts(100, 64, 32, 0, 5) == (0, 64) and O.block_parts(40, 64, 16, 5, 0) == (0, 0)
    assert O.block_parts(100, 16, 16, 1000, 0) == (96, 96)
    k = np.array([[1.0, math.nan, -math.inf, math.nan], [-2.0, 5.0, 3.0, math.nan]])
    lo, hi = O.block_bounds(k, 100.0)
    assert lo.tolist() == [-2, 5, -100, 0] and hi.tolist() == [1, 5, 3, 0]
    lo, hi = np.array([[0.0, 0], [-1, 2], [-1, 2]]), np.array([[1.0, 1], [1, 2], [1, 2]])
    q = np.array([[1.0, 1.0], [-3.0, 0.0]])                # scores: max(2, 0), max(3, 3), the same
    assert O.choose_blocks(q, lo, hi, 10, 1) == [11] and O.choose_blocks(q, lo, hi, 10, 2) == [11, 12] and O.choose_blocks(q, lo, hi, 10, 9) == [10, 11, 12]
    assert O.choose_blocks(q * math.nan, lo, hi, 0, 2) == [0, 1]
    sees = O.block_visible(6, 2, 1, 5, 2, [[1], []])
    assert sees.astype(int).tolist() == [[1, 0, 1, 1, 0, 1, 1, 0], [1, 0, 0, 0, 0, 1, 1, 1]]
