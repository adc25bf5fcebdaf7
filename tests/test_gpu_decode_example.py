"""The speculative decode step as it is used: examples/speculative_decode.py."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("nodes,branches", [(4, 1), (4, 3), (3, 2)])
def test_greedy_trees_give_the_tokens_of_one_at_a_time(dtype, nodes, branches):
    import speculative_decode as S
    prompts = [[1, 2, 3, 4, 5, 6, 7], [100, 90, 80]]
    one, one_steps = S.generate(S.Decoder(dtype=dtype, window=24, sinks=2), prompts, 40, nodes=1, greedy=True)
    out, steps = S.generate(S.Decoder(dtype=dtype, window=24, sinks=2), prompts, 40, nodes, branches, greedy=True)
    for o, x, p in zip(one, out, prompts):
        assert x[:len(p) + 40] == o[:len(p) + 40]
    assert steps <= one_steps


def test_sampling_runs_and_gives_pages_back():
    import speculative_decode as S
    import paper_2412_01380_amd as D
    m = S.Decoder(max_tokens=128)
    out, steps = S.generate(m, [[5, 6, 7, 8]] * 2, 50, 4, 2)
    assert all(len(o) >= 54 and 0 <= min(o) and max(o) < m.vocab for o in out)
    held = m.cache.page_refs.sum().item()
    assert held == sum(-(-n // 16) for n in m.lens) and m.cache.seq_len.tolist() == m.lens
    D.dip_kv_free(m.cache, m.seqs)
    assert not m.cache.page_refs.any()
