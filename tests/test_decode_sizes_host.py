"""Calls whose launches would have 2^32 threads and more, or whose rows do not fit 32 bits, are refused by name, before the
HIP runtime is touched."""
import ctypes as C

import pytest

from test_decode_host import FAKE, batch, cache


@pytest.fixture(scope="module")
def D():
    import paper_2412_01380_amd as D
    return D


def test_long_lists(D):
    L, c = D.lib, cache()
    r, n = C.byref(c), 1 << 24
    assert L.dip_kv_free(r, FAKE, n, None) == D.DIP_ERR_INVALID_ARG
    assert L.dip_kv_fork(r, FAKE, FAKE, n, None) == D.DIP_ERR_INVALID_ARG
    assert L.dip_kv_copy_pages(r, FAKE, FAKE, n, None) == D.DIP_ERR_INVALID_ARG
    assert "list" in D.dip_last_error()


def test_many_entries_beside_a_long_one(D):
    # 1024 entries that may have 60000 rows each: 2^32 threads in blocks of 256 rows and 512 threads
    c = cache(n_kv_heads=10, page_stride=16 * 10 * 128)
    b = batch(n_batch=1024, n_rows=100000, max_rows=60000)
    assert D.lib.dip_attention_workspace_bytes(C.byref(c), C.byref(b), 40, 0, 0) == 0
    st = D.lib.dip_window_attention(C.byref(c), 0, C.byref(b), FAKE, 5120, 40, 1.0, 0, 0, FAKE, 5120, FAKE, 1 << 40, None)
    assert st == D.DIP_ERR_UNSUPPORTED and "too many rows" in D.dip_last_error()
    # half as many fit
    b = batch(n_batch=1024, n_rows=100000, max_rows=30000)
    assert D.lib.dip_attention_workspace_bytes(C.byref(c), C.byref(b), 40, 0, 0) >= 256


def test_enormous_rows(D):
    # one position of all heads: 2^32 elements
    c, b = cache(dtype=0, n_kv_heads=65535, head_dim=65536, page_size=1, slot_stride=65536, head_stride=65536,
                 page_stride=65535 * 65536, layer_stride=9 * 65535 * 65536), batch()
    n = 65535 * 65536
    assert D.lib.dip_kv_append(C.byref(c), 0, 1, C.byref(b), FAKE, FAKE, n, n, None) == D.DIP_ERR_UNSUPPORTED
    assert D.lib.dip_kv_compact(C.byref(c), C.byref(b), FAKE, FAKE, None) == D.DIP_ERR_UNSUPPORTED
