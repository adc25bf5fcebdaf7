"""Calls of a decode step on two streams at once, each with a workspace of its own: the results of one after the other."""
import math

import pytest
import torch

from test_gpu_blocks import Long
from test_gpu_decode import ints, workspace
from test_gpu_sample import floats, logits

pytestmark = pytest.mark.gpu


def test_two_streams_at_once():
    import paper_2412_01380_amd as D
    rot = D.Rotary(D.dip_rotary_frequencies(128).cuda())
    jobs = []
    for seed in range(2):
        s = Long("bf16", [5000, 900, 64], [1, 1, 1], 8, 2, 128, 16, 16, seed=seed)
        s.update()
        x, u = logits(20, 50001, "f32", seed)
        q = s.q.cuda()
        how = dict(top_k=ints([50 + i for i in range(20)]), top_p=floats([0.9] * 20))
        jobs.append(dict(s=s, x=x, u=u, q=q, how=how, turned=torch.empty_like(q), blocks=torch.empty(3, 2, 20, dtype=torch.int32, device="cuda"),
                         out=torch.empty_like(q), token=torch.empty(20, dtype=torch.int32, device="cuda"), probs=torch.empty_like(x),
                         pos=ints([5000, 900, 64]),
                         ws=workspace(max(D.dip_select_blocks_workspace_bytes(s.cache, s.batch, 8, 16), D.dip_sample_workspace_bytes(20, 50001),
                                          D.dip_block_attention_workspace_bytes(s.cache, s.batch, 8, 16, 20, 4, 50)))))

    def go(j, stream):
        s = j["s"]
        D.dip_rotate_rows(rot, j["q"], j["pos"], j["turned"], stream)
        D.dip_kv_block_bounds(s.cache, s.layer, 1, s.seqs_dev, 0, s.bounds, stream)
        D.dip_select_blocks(s.cache, s.layer, s.batch, j["turned"], s.bounds, 4, 50, j["blocks"], j["ws"], stream)
        D.dip_block_attention(s.cache, s.layer, s.batch, None, j["blocks"], 16, j["turned"], 1 / math.sqrt(128), 4, 50, j["out"], j["ws"], stream)
        D.dip_sample(j["x"], j["u"], j["token"], j["probs"], j["ws"], stream=stream, **j["how"])

    results = []
    for j in jobs:
        go(j, None)
        torch.cuda.synchronize()
        results.append([j[k].clone() for k in ("turned", "blocks", "out", "token", "probs")])
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(5):
        for j in jobs:
            for k in ("turned", "blocks", "out", "token", "probs"):
                j[k].zero_()
        torch.cuda.synchronize()
        for _ in range(4):
            for j, st in zip(jobs, streams):
                go(j, st)
        torch.cuda.synchronize()
        for j, want in zip(jobs, results):
            assert all(torch.equal(j[k], w) for k, w in zip(("turned", "blocks", "out", "token", "probs"), want))
