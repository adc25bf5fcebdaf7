"""The calls of a decode step as a program runs them together: rows turned into the cache, blocks chosen and read, tokens
drawn, pages kept, forked, given back and their bounds kept up, against a model of the sequences in 64 bits."""
import math
import os
import sys

import numpy as np
import pytest
import torch

from oracle import decode_oracle as O
from test_gpu_decode import ints, starts, workspace

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

HQ, HKV, DIM, PAGE, BLOCK, LAYERS = 4, 2, 64, 32, 16, 2


class Run:
    def __init__(self, n_seqs=4, n_pages=64, max_pages=24, seed=0):
        import paper_2412_01380_amd as D
        self.D, self.g = D, torch.Generator().manual_seed(seed)
        kv = lambda: torch.full((LAYERS, n_pages, HKV, PAGE, DIM), float("nan"), device="cuda")
        self.cache = D.KvCache(kv(), kv(), ints([[0] * max_pages] * n_seqs), ints([0] * n_seqs), ints([0] * n_pages))
        D.dip_kv_init(self.cache)
        self.bounds = torch.full((LAYERS, n_pages, HKV, PAGE // BLOCK, 2, DIM), float("nan"), device="cuda")
        self.freq = D.dip_rotary_frequencies(DIM, kind=D.DIP_SCALING_LINEAR, factor=2.0)
        self.rot = D.Rotary(self.freq.cuda(), D.DIP_ROTARY_INTERLEAVED)
        self.text = [[] for _ in range(n_seqs)]                # per sequence the (keys, values) of its tokens, [LAYERS][HKV][DIM]

    def step(self, seqs, rows, parents=None, keep=None, path=None, sinks=3, recent=20, n_select=3):
        D = self.D
        n, lens = sum(rows), [len(self.text[s]) for s in seqs]
        batch = D.Batch(starts(rows), n, max(rows), seqs=ints(seqs), max_len=max(a + r for a, r in zip(lens, rows)))
        granted = ints([0] * len(seqs))
        D.dip_kv_reserve(self.cache, batch, granted, workspace(D.dip_kv_reserve_workspace_bytes(self.cache, batch)))
        assert all(granted.tolist())
        par = None if parents is None else ints([x for p in parents for x in p])
        ws = workspace(max(D.dip_select_blocks_workspace_bytes(self.cache, batch, HQ, BLOCK),
                           D.dip_block_attention_workspace_bytes(self.cache, batch, HQ, BLOCK, n_select, sinks, recent)))
        pos = [p for i, (a, r) in enumerate(zip(lens, rows)) for p in (O.tree_positions(a, parents[i]) if parents else range(a, a + r))]
        new = []
        for layer in range(LAYERS):
            x = torch.randn(n, HQ + 2 * HKV, DIM, generator=self.g)
            q, k, v = x.cuda().split([HQ, HKV, HKV], 1)
            q_out, out = torch.empty(n, HQ, DIM, device="cuda"), torch.empty(n, HQ, DIM, device="cuda")
            blocks = torch.empty(n, HKV, n_select, dtype=torch.int32, device="cuda")
            D.dip_kv_append_rotary(self.cache, layer, batch, par, self.rot, q, q_out, k, v)
            D.dip_select_blocks(self.cache, layer, batch, q_out, self.bounds, sinks, recent, blocks, ws)
            D.dip_block_attention(self.cache, layer, batch, par, blocks, BLOCK, q_out, DIM ** -0.5, sinks, recent, out, ws)
            q64 = O.turn(x[:, :HQ].double().numpy(), pos, self.freq.numpy(), True)
            k64 = O.turn(x[:, HQ:HQ + HKV].double().numpy(), pos, self.freq.numpy(), True)
            v64 = x[:, HQ + HKV:].double().numpy()
            new.append((k64, v64))
            at, g = 0, HQ // HKV
            for i, (s, a, r) in enumerate(zip(seqs, lens, rows)):
                front, tail = O.block_parts(a, PAGE, BLOCK, sinks, recent)
                for h in range(HKV):
                    keys = np.stack([t[0][layer][h] for t in self.text[s]] + [k64[at + t, h] for t in range(r)])
                    vals = np.stack([t[1][layer][h] for t in self.text[s]] + [v64[at + t, h] for t in range(r)])
                    lists = [blocks[at + t, h].tolist() for t in range(r)]
                    for t in range(r):                          # a good choice: no block left out scores higher than one taken
                        span = range(front // BLOCK, tail // BLOCK)
                        score = {}
                        for b in span:
                            lo, hi = O.block_bounds(keys[b * BLOCK:(b + 1) * BLOCK], 3e38)
                            qq = q64[at + t, h * g:(h + 1) * g]
                            score[b] = (np.maximum(qq, 0) * hi + np.minimum(qq, 0) * lo).sum(1).max()
                        took = [b for b in lists[t] if b >= 0]
                        assert len(took) == min(n_select, len(span)) and set(took) <= set(span)
                        left = [score[b] for b in span if b not in took]
                        # (the cache holds fp32 keys: 14 roundings of 2^-24 of |k| <= 8, over 64 dims of |q| <= 8)
                        assert not left or max(left) <= min(score[b] for b in took) + 14 * 2.0 ** -24 * 8 * 64 * 8
                    sees = O.block_visible(a, r, front, tail, BLOCK, [[b for b in x if b >= 0] for x in lists], parents[i] if parents else None)
                    ref, _, _ = O.attend(q64[at:at + r, h * g:(h + 1) * g], keys[:, None], vals[:, None], sees, DIM ** -0.5)
                    err = np.abs(out[at:at + r, h * g:(h + 1) * g].double().cpu().numpy() - ref).max()
                    assert err <= 2e-5, err                      # (fp32 throughout: scores of some 10, 300 of their roundings)
                at += r
        D.dip_kv_compact(self.cache, batch, None if path is None else ints([x for p, r in zip(path, rows) for x in p + [-1] * (r - len(p))]),
                         None if keep is None else ints(keep))
        D.dip_kv_block_bounds(self.cache, 0, LAYERS, ints(seqs), max(rows), self.bounds)
        at = 0
        for i, (s, r) in enumerate(zip(seqs, rows)):
            kept = (path[i] if path else list(range(r)))[:keep[i] if keep else r]
            self.text[s] += [tuple([new[layer][w][at + t] for layer in range(LAYERS)] for w in range(2)) for t in kept]
            at += r
        assert self.cache.seq_len.tolist() == [len(t) for t in self.text]


def test_prompts_tokens_trees_and_branches():
    run = Run()
    run.step([0, 1], [200, 33])
    run.step([0, 1], [1, 1])
    run.D.dip_kv_fork(run.cache, ints([0, 0]), ints([2, 3]))   # branches share pages and their bounds; the last one is copied on write
    run.text[2], run.text[3] = list(run.text[0]), list(run.text[0])
    run.step([2, 3, 0], [1, 1, 1])
    tree = [-1, 0, 0, 1, 2, 3]
    run.step([3, 1, 2], [6, 6, 6], [tree] * 3, [3, 1, 4], [[0, 1, 3], [0], [0, 1, 3, 5]])
    for i in range(12):                                        # across the ends of pages
        run.step([1, 2, 3], [1, 5, 3], [[-1], [-1, 0, 1, 2, 3], [-1, 0, 0]], [1, 1 + i % 5, 2], [[0], list(range(1 + i % 5)), [0, 2]])
    run.D.dip_kv_free(run.cache, ints([0, 3]))
    run.text[0], run.text[3] = [], []
    run.step([0, 2], [70, 1], n_select=1, sinks=0, recent=0)   # pages that were others' a moment ago
    run.step([0, 2], [1, 40], n_select=9)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_greedy_trees_over_chosen_blocks_give_the_tokens_of_one_at_a_time(dtype):
    import speculative_decode as S
    prompts = [list(range(1, 120)), [100, 90, 80]]
    # a window of all, and blocks enough to hold all: what is read does not hang on how far the pages are filled
    make = lambda: S.Decoder(dtype=dtype, blocks=40, sinks=2, recent=8)
    one, _ = S.generate(make(), prompts, 40, nodes=1, greedy=True)
    out, _ = S.generate(make(), prompts, 40, 4, 2, greedy=True)
    full, _ = S.generate(S.Decoder(dtype=dtype, window=0), prompts, 40, 4, 2, greedy=True)
    for o, x, f, p in zip(one, out, full, prompts):
        assert x[:len(p) + 40] == o[:len(p) + 40] == f[:len(p) + 40]


def test_sampling_over_few_blocks_runs_and_gives_pages_back():
    import speculative_decode as S
    import paper_2412_01380_amd as D
    m = S.Decoder(max_tokens=256, blocks=2, recent=10)
    out, _ = S.generate(m, [list(range(5, 90))] * 2, 50, 4, 2)
    assert all(len(o) >= 135 and 0 <= min(o) and max(o) < m.vocab for o in out)
    D.dip_kv_free(m.cache, m.seqs)
    assert not m.cache.page_refs.any()
