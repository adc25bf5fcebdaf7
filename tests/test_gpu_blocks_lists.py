"""Attention over lists of blocks of a caller's own making: what is passed over costs nothing that stands behind it, wherever
in a list, few or many, and in contexts of fewer blocks than a list has entries."""
import math

import numpy as np
import pytest
import torch

from oracle import decode_oracle as O
from test_gpu_blocks import Long
from test_gpu_decode import ints

pytestmark = pytest.mark.gpu


def named(lists, lo, hi):
    """The entries that are read: in [lo, hi), and above the one before."""
    return [[b for i, b in enumerate(x) if lo <= b < hi and (i == 0 or b > x[i - 1])] for x in lists]


def padded(lists):
    want = torch.full((len(lists), 2, max(1, max(map(len, lists)))), -1)
    for r, x in enumerate(lists):
        want[r, :, :len(x)] = torch.tensor(x, dtype=want.dtype)
    return want


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("given", [
    [0, 1, 2, 3], [-1, 1, 2, 3], [0, 0, -7, 1, 2, 99, 3], [1, 1, 1, 2, 2, 2, 3, 3, 3], [3, 2, 1], [9, 0, 3], [-1, -1, -1, -1], [2, -1, 3, -1, -1],
    [99, 98, 97, 96, 95, 94, 3], [1, 2, 3, -1, -1, -1, -1, -1], list(range(-70, 5)), [-1] * 200 + [1] + [0] * 63 + [2, 3], [-1] * 4095 + [2]])
def test_what_is_passed_over_pushes_nothing_out(given, dtype):
    s = Long(dtype, [400, 90], [2, 1], 8, 2, 128, 16, 16)      # sinks 5, recent 20: blocks 1 .. 22 of entry 0, 1 .. 3 of entry 1
    blocks = ints([[given, given]] * 3).contiguous()
    read = named([given, given], 1, 23) + named([given], 1, 4)
    s.check_attention(s.attend(blocks, 5, 20), padded(read), 5, 20)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page,block", [(64, 16, 16), (96, 64, 32), (128, 128, 64)])
def test_gaps_in_lists_of_several_shares(d, page, block, dtype):
    # every kind of entry that is passed over, between valid ones, in lists far longer than the context has blocks
    rng = np.random.default_rng(d)
    s = Long(dtype, [6000, 1500, 40], [1, 2, 1], 10, 2, d, page, block, d == 96, seed=3)
    parts = [O.block_parts(n, page, block, 70, 100) for n in s.lens for _ in range(2 if n == 1500 else 1)]
    lists = []
    for front, tail in parts:
        x, b = [], front // block
        while len(x) < 900:
            kind = rng.integers(0, 5)
            if kind == 0:
                x.append(int(rng.integers(-3, front // block)))
            elif kind == 1:
                x.append(int(x[-1]) if x else -1)
            elif kind == 2 and rng.random() < 0.1:
                x.append(10 ** 6 + len(x))
            elif b < tail // block:
                x.append(b)
                b += 1 + int(rng.integers(0, 2))
            else:
                x.append(-1)
        lists.append(x)
    blocks = ints([[x, x] for x in lists]).contiguous()
    read = [named([x], f // block, t // block)[0] for x, (f, t) in zip(lists, parts)]
    assert len(read[0]) > 40
    s.check_attention(s.attend(blocks, 70, 100), padded(read), 70, 100)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_choice_with_fewer_sinks_than_the_attention(dtype):
    s = Long(dtype, [700, 130], [2, 3], 8, 2, 64, 16, 16)
    s.update()
    blocks = s.select(60, 0, 20)                               # all of them, the first ones too
    front = [O.block_parts(n, 16, 16, 75, 20) for n in (700, 130)]
    read = [list(range(f // 16, t // 16)) for f, t in [front[0]] * 2 + [front[1]] * 3]
    s.check_attention(s.attend(blocks, 75, 20), padded(read), 75, 20)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_block_that_a_list_names_again_and_again(dtype):
    # behind a smaller entry a block is above the one before it, and is read once more: here far more often than the context is long
    s = Long(dtype, [3000], [1], 4, 2, 128, 16, 16, seed=9)
    for times in (2, 1500):
        blocks = ints([[[5, 3] * times] * 2]).contiguous()
        got = s.attend(blocks, 0, 20)[0].double().cpu().numpy()
        front, tail = O.block_parts(3000, 16, 16, 0, 20)
        at = list(range(front)) + list(range(80, 96)) * times + list(range(tail, 3001))
        for h in range(2):
            ref, mag, big = O.attend(s.q64[:, 2 * h:2 * h + 2], s.k[0][at, h:h + 1], s.v[0][at, h:h + 1], np.ones((1, len(at)), bool), 1 / math.sqrt(128))
            dz = (big * (128 / 4 + 8) + 64)[..., None] * 2.0 ** -24
            bound = mag * (2 * dz + (4 * math.sqrt(len(at)) + 32) * 2.0 ** -24) + 1e-30
            if dtype == "bf16":
                bound = bound + mag * 2.0 ** -14 + np.abs(ref) * 2.0 ** -8
            assert (np.abs(got[2 * h:2 * h + 2] - ref[0]) <= bound[0]).all(), times


def test_lists_of_different_lengths_in_a_graph():
    import paper_2412_01380_amd as D
    s = Long("bf16", [3000, 90], [1, 1], 8, 2, 128, 16, 16)
    q, blocks = s.q.cuda(), torch.empty(2, 2, 300, dtype=torch.int32, device="cuda")
    ws = torch.empty(D.dip_block_attention_workspace_bytes(s.cache, s.batch, 8, 16, 300, 5, 20), dtype=torch.uint8, device="cuda")
    out, graph = torch.empty_like(q), torch.cuda.CUDAGraph()
    blocks.fill_(-1)
    with torch.cuda.graph(graph):
        D.dip_block_attention(s.cache, s.layer, s.batch, None, blocks, 16, q, 1 / math.sqrt(128), 5, 20, out, ws)
    for lists in ([[0, 1, 2, 3], [-1, 1, 2, 3]], [list(range(-100, 190)), [-1] * 299 + [3]], [[-1], [-1]], [[], list(range(4))]):
        blocks.fill_(-1)
        for r, x in enumerate(lists):
            blocks[r, :, :len(x)] = ints(x)
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        read = named([lists[0]], 1, O.block_parts(3000, 16, 16, 5, 20)[1] // 16) + named([lists[1]], 1, 4)
        s.check_attention(out, padded(read), 5, 20)
        assert torch.equal(out, s.attend(blocks, 5, 20, ws=ws))
