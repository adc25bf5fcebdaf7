"""Host-side checks of the calls around the MLP, without a GPU: bad arguments are refused before the HIP
runtime is touched, workspaces have sizes, and the 64-bit oracle agrees with hand-worked cases."""
import ctypes as C

import numpy as np
import pytest

from oracle import decode_oracle as O

FAKE = 0x10000    # a non-null, 256-aligned "device pointer"; validation never dereferences it


@pytest.fixture(scope="module")
def D():
    import paper_2412_01380_amd as D
    return D


def cache(**over):
    from paper_2412_01380_amd.libdip import _KvCache
    f = dict(k=FAKE, v=FAKE, page_table=FAKE, seq_len=FAKE, page_refs=FAKE, dtype=1, n_layers=2, n_pages=9, page_size=16,
             n_kv_heads=2, head_dim=128, n_seqs=3, max_pages=4, layer_stride=9 * 16 * 256, page_stride=16 * 256,
             head_stride=16 * 128, slot_stride=128)
    f.update(over)
    return _KvCache(*[f[n] for n, _ in _KvCache._fields_])


def batch(**over):
    from paper_2412_01380_amd.libdip import _Batch
    f = dict(seqs=FAKE, row_start=FAKE, n_batch=2, n_rows=5, max_rows=3, max_len=0)
    f.update(over)
    return _Batch(*[f[n] for n, _ in _Batch._fields_])


BAD_CACHES = [
    (dict(k=None), "INVALID_ARG"), (dict(v=None), "INVALID_ARG"), (dict(page_table=None), "INVALID_ARG"),
    (dict(seq_len=None), "INVALID_ARG"), (dict(page_refs=None), "INVALID_ARG"), (dict(dtype=2), "UNSUPPORTED"),
    (dict(n_layers=0), "INVALID_ARG"), (dict(n_pages=0), "INVALID_ARG"), (dict(n_seqs=-1), "INVALID_ARG"),
    (dict(max_pages=0), "INVALID_ARG"), (dict(page_size=0), "UNSUPPORTED"), (dict(page_size=24), "UNSUPPORTED"),
    (dict(page_size=8192), "UNSUPPORTED"), (dict(max_pages=1 << 28), "UNSUPPORTED"), (dict(head_dim=12), "UNSUPPORTED"),
    (dict(slot_stride=129), "UNSUPPORTED"), (dict(slot_stride=64), "INVALID_ARG"), (dict(page_stride=8), "INVALID_ARG"),
    (dict(layer_stride=0), "INVALID_ARG"), (dict(k=FAKE + 8), "UNSUPPORTED"),
]


@pytest.mark.parametrize("over,status", BAD_CACHES)
def test_caches_are_refused(D, over, status):
    L, c, b = D.lib, cache(**over), batch()
    want = getattr(D, "DIP_ERR_" + status)
    r, rb = C.byref(c), C.byref(b)
    assert L.dip_kv_init(r, None) == want
    assert L.dip_kv_free(r, FAKE, 1, None) == want
    assert L.dip_kv_fork(r, FAKE, FAKE, 1, None) == want
    assert L.dip_kv_copy_pages(r, FAKE, FAKE, 1, None) == want
    assert L.dip_kv_reserve(r, rb, None, FAKE, 1 << 30, None) == want
    assert L.dip_kv_append(r, 0, 1, rb, FAKE, FAKE, 256, 0, None) == want
    assert L.dip_kv_compact(r, rb, FAKE, FAKE, None) == want
    assert L.dip_window_attention(r, 0, rb, FAKE, 512, 4, 1.0, 0, 0, FAKE, 512, FAKE, 1 << 30, None) == want
    assert L.dip_kv_reserve_workspace_bytes(r, rb) == 0
    assert L.dip_attention_workspace_bytes(r, rb, 4, 0, 0) == 0
    assert "cache" in D.dip_last_error()


BAD_BATCHES = [
    (dict(seqs=None), "INVALID_ARG"), (dict(row_start=None), "INVALID_ARG"), (dict(n_batch=0), "UNSUPPORTED"),
    (dict(n_batch=1025), "UNSUPPORTED"), (dict(n_rows=0), "INVALID_ARG"), (dict(max_rows=0), "INVALID_ARG"),
    (dict(max_len=-1), "INVALID_ARG"), (dict(n_rows=1 << 24), "UNSUPPORTED"),
]


@pytest.mark.parametrize("over,status", BAD_BATCHES)
def test_batches_are_refused(D, over, status):
    L, c, b = D.lib, cache(), batch(**over)
    want = getattr(D, "DIP_ERR_" + status)
    r, rb = C.byref(c), C.byref(b)
    assert L.dip_kv_reserve(r, rb, None, FAKE, 1 << 30, None) == want
    assert L.dip_kv_append(r, 0, 1, rb, FAKE, FAKE, 256, 0, None) == want
    assert L.dip_kv_compact(r, rb, FAKE, FAKE, None) == want
    assert L.dip_window_attention(r, 0, rb, FAKE, 512, 4, 1.0, 0, 0, FAKE, 512, FAKE, 1 << 30, None) == want
    if "seqs" not in over:
        assert L.dip_verify_tree(rb, FAKE, FAKE, FAKE, 100, FAKE, 100, 0, 100, FAKE, FAKE, 2, FAKE, FAKE, FAKE, FAKE, 1 << 30,
                                 None) == want


def test_attention_arguments_are_refused(D):
    L = D.lib

    def call(c=None, b=None, layer=0, q=FAKE, qs=512, heads=4, scale=0.1, window=0, sinks=0, out=FAKE, os=512, ws=FAKE, n=1 << 30,
             tree=False, parents=FAKE):
        c, b = c or cache(), b or batch()
        if tree:
            return L.dip_tree_attention(C.byref(c), layer, C.byref(b), parents, q, qs, heads, scale, window, sinks, out, os, ws, n, None)
        return L.dip_window_attention(C.byref(c), layer, C.byref(b), q, qs, heads, scale, window, sinks, out, os, ws, n, None)

    for tree in (False, True):
        assert call(tree=tree, c=cache(head_dim=80, slot_stride=80)) == D.DIP_ERR_UNSUPPORTED
        assert call(tree=tree, layer=2) == D.DIP_ERR_INVALID_ARG
        assert call(tree=tree, layer=-1) == D.DIP_ERR_INVALID_ARG
        assert call(tree=tree, q=None) == D.DIP_ERR_INVALID_ARG
        assert call(tree=tree, out=None) == D.DIP_ERR_INVALID_ARG
        assert call(tree=tree, heads=3, qs=384, os=384) == D.DIP_ERR_INVALID_ARG
        assert call(tree=tree, heads=0) == D.DIP_ERR_INVALID_ARG
        assert call(tree=tree, qs=504) == D.DIP_ERR_INVALID_ARG
        assert call(tree=tree, os=516) == D.DIP_ERR_UNSUPPORTED
        assert call(tree=tree, q=FAKE + 2) == D.DIP_ERR_UNSUPPORTED
        assert call(tree=tree, window=-1) == D.DIP_ERR_INVALID_ARG
        assert call(tree=tree, sinks=-1) == D.DIP_ERR_INVALID_ARG
        for scale in (0.0, -1.0, float("nan"), float("inf")):
            assert call(tree=tree, scale=scale) == D.DIP_ERR_INVALID_ARG
        assert call(tree=tree, ws=None) == D.DIP_ERR_WORKSPACE
        assert call(tree=tree, ws=FAKE + 16) == D.DIP_ERR_WORKSPACE
        assert call(tree=tree, n=255) == D.DIP_ERR_WORKSPACE
    assert call(tree=True, parents=None) == D.DIP_ERR_INVALID_ARG
    assert call(tree=True, b=batch(n_rows=100, max_rows=65)) == D.DIP_ERR_UNSUPPORTED


def test_workspaces_cover_every_shape(D):
    for dtype, dims in ((1, 128), (0, 96)):
        for rows in (1, 8, 64, 5000):
            for n in (1, 7, 1024):
                c = cache(dtype=dtype, head_dim=dims, slot_stride=dims)
                b = batch(n_batch=n, n_rows=max(rows, n), max_rows=rows)
                need = D.lib.dip_attention_workspace_bytes(C.byref(c), C.byref(b), 8, 100, 4)
                assert 256 <= need <= 64 << 20
                assert D.lib.dip_kv_reserve_workspace_bytes(C.byref(c), C.byref(b)) >= 256


def test_page_calls_refuse_their_own_arguments(D):
    L, c, b = D.lib, cache(), batch()
    r, rb = C.byref(c), C.byref(b)
    assert L.dip_kv_free(r, None, 1, None) == D.DIP_ERR_INVALID_ARG
    assert L.dip_kv_free(r, FAKE, 0, None) == D.DIP_ERR_INVALID_ARG
    assert L.dip_kv_fork(r, FAKE, None, 1, None) == D.DIP_ERR_INVALID_ARG
    assert L.dip_kv_copy_pages(r, FAKE, FAKE, -1, None) == D.DIP_ERR_INVALID_ARG
    need = L.dip_kv_reserve_workspace_bytes(r, rb)
    assert L.dip_kv_reserve(r, rb, None, FAKE, need - 1, None) == D.DIP_ERR_WORKSPACE
    assert L.dip_kv_reserve(r, rb, None, None, need, None) == D.DIP_ERR_WORKSPACE
    append = lambda layer=0, n=1, k=FAKE, v=FAKE, rs=256, ls=0: L.dip_kv_append(r, layer, n, rb, k, v, rs, ls, None)
    assert append(layer=2) == D.DIP_ERR_INVALID_ARG
    assert append(layer=1, n=2, ls=2048) == D.DIP_ERR_INVALID_ARG
    assert append(n=0) == D.DIP_ERR_INVALID_ARG
    assert append(k=None) == D.DIP_ERR_INVALID_ARG
    assert append(rs=248) == D.DIP_ERR_INVALID_ARG
    assert append(rs=260) == D.DIP_ERR_UNSUPPORTED
    assert append(n=2, ls=0) == D.DIP_ERR_INVALID_ARG
    assert append(v=FAKE + 4) == D.DIP_ERR_UNSUPPORTED


def test_verify_arguments_are_refused(D):
    L = D.lib

    def call(b=None, ps=100, qs=100, dtype=0, vocab=100, kids=2, n=1 << 30, ws=FAKE, **null):
        b = b or batch()
        a = dict(tokens=FAKE, parents=FAKE, p=FAKE, q=FAKE, u=FAKE, us=FAKE, keep=FAKE, path=FAKE, token=FAKE)
        a.update(null)
        return L.dip_verify_tree(C.byref(b), a["tokens"], a["parents"], a["p"], ps, a["q"], qs, dtype, vocab, a["u"], a["us"], kids,
                                 a["keep"], a["path"], a["token"], ws, n, None)

    for name in ("tokens", "parents", "p", "q", "u", "us", "keep", "path", "token"):
        assert call(**{name: None}) == D.DIP_ERR_INVALID_ARG
    assert call(ps=99) == D.DIP_ERR_INVALID_ARG
    assert call(qs=99) == D.DIP_ERR_INVALID_ARG
    assert call(dtype=2) == D.DIP_ERR_UNSUPPORTED
    assert call(vocab=0) == D.DIP_ERR_INVALID_ARG
    assert call(vocab=(1 << 24) + 1, ps=1 << 25, qs=1 << 25) == D.DIP_ERR_UNSUPPORTED
    assert call(kids=0) == D.DIP_ERR_INVALID_ARG
    assert call(kids=64) == D.DIP_ERR_INVALID_ARG
    assert call(p=FAKE + 2) == D.DIP_ERR_UNSUPPORTED
    assert call(b=batch(n_rows=70, max_rows=65)) == D.DIP_ERR_UNSUPPORTED
    assert call(ws=None) == D.DIP_ERR_WORKSPACE
    assert call(n=8) == D.DIP_ERR_WORKSPACE


# ---- the oracle on cases worked by hand ------------------------------------------------------------------
def test_oracle_visibility():
    v = O.visible(4, 2, 2, 1)
    assert v.astype(int).tolist() == [[1, 0, 0, 1, 1, 0], [1, 0, 0, 0, 1, 1]]
    t = O.visible(3, 4, 2, 0, [-1, 0, 0, 2])          # node 3: depth 2, stands at 5, sees no committed position
    assert t.astype(int).tolist() == [[0, 0, 1, 1, 0, 0, 0], [0, 0, 0, 1, 1, 0, 0], [0, 0, 0, 1, 0, 1, 0], [0, 0, 0, 1, 0, 1, 1]]
    assert O.ancestors([-1, 5, 1, 0, -7]) == [[0], None, None, [0, 3], None]


def test_oracle_attention_against_a_dense_softmax():
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(3, 4, 8)), rng.normal(size=(7, 2, 8)), rng.normal(size=(7, 2, 8))
    sees = O.visible(4, 3, 0, 0)
    out, _, _ = O.attend(q, k, v, sees, 0.3)
    for t in range(3):
        for h in range(4):
            z = np.where(sees[t], 0.3 * k[:, h // 2] @ q[t, h], -np.inf)
            p = np.exp(z - z.max()) / np.exp(z - z.max()).sum()
            assert np.allclose(out[t, h], p @ v[:, h // 2], atol=1e-12)


def test_oracle_verification_is_lossless_on_a_tiny_vocabulary():
    # one child, every draft and a fine grid of numbers: the distribution of the token behind node 0 is the target's
    p, q = np.array([[0.5, 0.3, 0.2]] * 2), np.array([[0.2, 0.2, 0.6]] * 2)
    n, got = 200, np.zeros(3)
    for x in range(3):
        for i in range(n):
            path, tok = O.verify([-1, 0], [0, x], p, q, [0.0, (i + 0.5) / n], 0.0, 1)
            if len(path) == 2:
                got[x] += q[0, x] / n
            else:
                for j in range(n):
                    got[O.verify([-1, 0], [0, x], p, q, [0.0, (i + 0.5) / n], (j + 0.5) / n, 1)[1]] += q[0, x] / n / n
    assert np.allclose(got, p[0], atol=0.01)


def test_oracle_pool_by_hand():
    o = O.Pool(6, 4, 3, 4)
    assert o.reserve([0], [6]) == [1] and o.table[0] == [0, 1, -1, -1]
    o.append([0], [list("abcdef")])
    o.compact([0], [6], None, None)
    o.fork([0], [2])
    assert o.refs == [2, 2, 0, 0, 0, 0]
    assert o.reserve([2], [3]) == [1] and o.table[2] == [0, 2, 3, -1] and o.refs == [2, 1, 1, 1, 0, 0]
    assert o.rows[2, 0] == "e" and o.rows[2, 1] == "f"
    o.append([2], [list("xyz")])
    o.compact([2], [3], [[0, 2]], [2])
    assert o.len == [6, 0, 8] and o.table[2] == [0, 2, -1, -1] and o.rows[2, 3] == "z"
    o.free([0, 2])
    assert o.refs == [0] * 6


def test_longest_tables(D):
    """A length and a step's rows on top of it fit 32 bits: tables end 2^25 positions before that."""
    b = batch()
    longest = cache(max_pages=(1 << 27) - (1 << 21))
    assert D.lib.dip_attention_workspace_bytes(C.byref(longest), C.byref(b), 4, 0, 0) > 0
    assert D.lib.dip_attention_workspace_bytes(C.byref(cache(max_pages=longest.max_pages + 1)), C.byref(b), 4, 0, 0) == 0
    assert D.lib.dip_kv_reserve(C.byref(cache(max_pages=1 << 27)), C.byref(b), None, FAKE, 1 << 30, None) == D.DIP_ERR_UNSUPPORTED
