"""Views that torch counts as contiguous although a dimension of one entry has a stride of its own."""
import numpy as np
import pytest
import torch

from test_gpu_decode import Setup, check_verify, ints, starts, verify_inputs, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_row_out_of_heads_before_rows(dtype):
    import paper_2412_01380_amd as D
    s = Setup(dtype, [50], [1], 8, 2, 64, 16)
    q = s.q.cuda().view(8, 1, 64).transpose(0, 1)                      # [1][8][64], strides (64, 64, 1)
    out = torch.empty(8, 1, 64, dtype=q.dtype, device="cuda").transpose(0, 1)
    assert q.stride() == out.stride() == (64, 64, 1)
    s.check(s.run(0, 0, q=q, out=out))
    # the same row's key and value, written again, k and v of different strides in the dimension of one
    page, slot = int(s.table[s.seqs[0], 3]), 50 % 16
    k, v = s.cache.k[1, page, :, slot].clone()[:, None], s.cache.v[1, page, :, slot].clone()[None]
    s.cache.page_refs.fill_(1)
    s.cache.k[1, page, :, slot], s.cache.v[1, page, :, slot] = 0, 0
    D.dip_kv_append(s.cache, 1, s.batch, k.transpose(0, 1), v)
    s.check(s.run(0, 0))
    s.cache.k[1, page, :, slot], s.cache.v[1, page, :, slot] = 0, 0
    D.dip_kv_append(s.cache, 1, s.batch, k.transpose(0, 1)[None], v[None])
    s.check(s.run(0, 0))


def test_caches_of_one_layer_head_or_slot():
    import paper_2412_01380_amd as D
    g = torch.Generator(device="cuda").manual_seed(0)
    new = torch.randn(2, 5, 1, 64, generator=g, device="cuda")
    for page in (1, 4):
        k = torch.zeros(1, 9, 1, page, 64, device="cuda")
        v = torch.zeros(1, 9, 1, page, 64, device="cuda").as_strided((1, 9, 1, page, 64), (8, 64 * page, 8, 64, 1))
        cache = D.KvCache(k, v, ints([[-1] * 6]), ints([0]), ints([0] * 9))
        b = D.Batch(starts([5]), 5, 5, seqs=ints([0]))
        D.dip_kv_reserve(cache, b, None, workspace(D.dip_kv_reserve_workspace_bytes(cache, b)))
        D.dip_kv_append(cache, 0, b, new[0], new[1])
        D.dip_kv_compact(cache, b, None, None)
        table = cache.page_table[0].tolist()
        for r in range(5):
            assert torch.equal(k[0, table[r // page], :, r % page], new[0, r]) and torch.equal(v[0, table[r // page], :, r % page], new[1, r])


def test_verification_of_a_single_node():
    rng = np.random.default_rng(0)
    p, q, tokens, u, us = verify_inputs(rng, [[-1]], 500)
    p, q = (t.cuda().view(500, 1).t() for t in (p, q))                 # strides (1, 1)
    check_verify([[-1]], p, q, tokens, u, us, 1)
