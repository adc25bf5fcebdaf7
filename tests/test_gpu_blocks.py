"""Bounds of blocks, the choice among them and the attention over them against the 64-bit oracle: head layouts, page and block
sizes, lengths from nothing to long, trees, ties, lists of a caller's own making, and whatever lies in places that nobody
reads."""
import math

import numpy as np
import pytest
import torch

from oracle import decode_oracle as O
from test_gpu_decode import DT, NAN, Setup, ints, random_tree, workspace

pytestmark = pytest.mark.gpu

MOST = {"f32": float(torch.finfo(torch.float32).max), "bf16": float(torch.finfo(torch.bfloat16).max)}


class Long(Setup):
    """Setup with bounds, choices and the attention over them."""

    def __init__(self, dtype, lens, rows, hq, hkv, d, page, block, slot_major=False, seed=0, **kw):
        super().__init__(dtype, lens, rows, hq, hkv, d, page, slot_major, seed=seed, **kw)
        self.page, self.block = page, block
        k = self.cache.k
        self.bounds = torch.full((k.shape[0], k.shape[1], hkv, page // block, 2, d), 7.0, dtype=k.dtype, device="cuda")
        self.seqs_dev = ints(self.seqs)

    def update(self, back=0, layer=None, n_layers=1):
        import paper_2412_01380_amd as D
        D.dip_kv_block_bounds(self.cache, self.layer if layer is None else layer, n_layers, self.seqs_dev, back, self.bounds)

    def want_bounds(self, back=0):
        want = torch.full(self.bounds.shape, 7.0, dtype=torch.float64)
        for e, n in enumerate(self.lens):
            for j in range((max(0, n - back) if back else 0) // self.page, n // self.page):
                pg = int(self.table[self.seqs[e], j])
                for h in range(self.hkv):
                    for b in range(self.page // self.block):
                        at = j * self.page + b * self.block
                        lo, hi = O.block_bounds(self.k[e][at:at + self.block, h], MOST[self.dtype])
                        want[self.layer, pg, h, b, 0], want[self.layer, pg, h, b, 1] = torch.from_numpy(lo), torch.from_numpy(hi)
        return want

    def select(self, n_select, sinks, recent, q=None):
        import paper_2412_01380_amd as D
        out = torch.full((len(self.q), self.hkv, n_select), -9, dtype=torch.int32, device="cuda")
        ws = workspace(D.dip_select_blocks_workspace_bytes(self.cache, self.batch, self.hq, self.block))
        D.dip_select_blocks(self.cache, self.layer, self.batch, self.q.cuda() if q is None else q, self.bounds, sinks, recent, out, ws)
        return out

    def want_choice(self, n_select, sinks, recent):
        want, at, g = np.full((len(self.q), self.hkv, n_select), -1), 0, self.hq // self.hkv
        for e, (n, r) in enumerate(zip(self.lens, self.rows)):
            front, tail = O.block_parts(n, self.page, self.block, sinks, recent)
            blocks = range(front // self.block, tail // self.block)
            for h in range(self.hkv if len(blocks) else 0):
                lo, hi = (np.stack(x) for x in zip(*[O.block_bounds(self.k[e][b * self.block:(b + 1) * self.block, h], MOST[self.dtype]) for b in blocks]))
                for t in range(r):
                    got = O.choose_blocks(self.q64[at + t, h * g:(h + 1) * g], lo, hi, front // self.block, n_select)
                    want[at + t, h, :len(got)] = got
            at += r
        return want

    def attend(self, blocks, sinks, recent, parents=None, q=None, out=None, ws=None, batch=None):
        import paper_2412_01380_amd as D
        q = self.q.cuda() if q is None else q
        b = batch or self.batch
        out = torch.full((len(q), self.hq, self.d), NAN, dtype=q.dtype, device="cuda") if out is None else out
        ws = workspace(D.dip_block_attention_workspace_bytes(self.cache, b, self.hq, self.block, blocks.shape[-1], sinks, recent)) if ws is None else ws
        par = None if parents is None else ints([x for p in parents for x in p])
        D.dip_block_attention(self.cache, self.layer, b, par, blocks, self.block, q, 1 / math.sqrt(self.d), sinks, recent, out, ws)
        return out

    def check_attention(self, out, chosen, sinks, recent, parents=None, max_len=None):
        """As Setup.check: fp32 scores and sums, two terms to a bf16 weight, the output rounded once."""
        got, at, g = out.double().cpu().numpy(), 0, self.hq // self.hkv
        for e, (n, r) in enumerate(zip(self.lens, self.rows)):
            front, tail = O.block_parts(min(n, max_len or n), self.page, self.block, sinks, recent)
            for h in range(self.hkv):
                lists = [[b for b in chosen[at + t, h].tolist() if b >= 0] for t in range(r)]
                sees = O.block_visible(n, r, front, tail, self.block, lists, None if parents is None else parents[e])
                if max_len is not None:
                    sees[:, max_len:] = False
                heads = slice(h * g, (h + 1) * g)
                # (what nobody sees may be anything; the oracle must not multiply it by nothing)
                ref, mag, big = O.attend(self.q64[at:at + r, heads], self.k[e][:, h:h + 1], self.v[e][:, h:h + 1], sees, 1 / math.sqrt(self.d))
                dz = (big * (self.d / 4 + 8) + 64)[..., None] * 2.0 ** -24
                bound = mag * (2 * dz + (4 * math.sqrt(n + r) + 32) * 2.0 ** -24) + 1e-30
                if self.dtype == "bf16":
                    bound = bound + mag * 2.0 ** -14 + np.abs(ref) * 2.0 ** -8
                err = np.abs(got[at:at + r, heads] - ref)
                assert np.isfinite(got[at:at + r, heads]).all(), (e, h)
                assert (err <= bound).all(), (e, h, float((err / bound).max()))
            at += r


CASES = [
    # lens, rows, hq, hkv, d, page, block, slot_major
    ([0], [1], 1, 1, 64, 16, 16, False),                       # the first token of all
    ([0, 5, 33], [1, 1, 1], 4, 2, 128, 16, 16, True),
    ([127, 128, 129, 300], [1] * 4, 8, 8, 96, 64, 32, False),
    ([1500, 3, 700], [1, 1, 1], 32, 4, 128, 16, 16, False),    # eight query heads share one
    ([511, 0, 40], [3, 20, 0], 10, 2, 64, 32, 16, True),       # an entry without rows
    ([1000, 65], [7, 9], 34, 2, 128, 128, 64, False),          # seventeen heads on one: more than a product's columns
    ([4000, 2100], [1, 2], 3, 1, 96, 128, 16, True),           # long enough for shares
    ([2600], [1], 5, 5, 64, 4096, 32, False),                  # a page that is never complete
    ([900, 1024], [2, 1], 6, 3, 128, 256, 256, True),
]
CHOICES = [(1, 0, 0), (3, 4, 20), (16, 33, 100), (200, 1, 0), (8, 0x7fffffff, 0), (8, 0, 0x7fffffff)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_bounds(case, dtype):
    lens, rows, hq, hkv, d, page, block, slot_major = CASES[case]
    for back in (0, 1, 17, page, 3 * page + 1, 10 ** 9):
        s = Long(dtype, lens, rows, hq, hkv, d, page, block, slot_major, seed=case)
        s.update(back)
        assert torch.equal(s.bounds.double().cpu(), s.want_bounds(back))
    # all layers at once, a sequence twice and numbers that are none
    s.seqs_dev = ints(s.seqs + s.seqs[:1] + [-1, 1000])
    s.layer, other = 0, s.bounds.clone()
    s.update(0, layer=0, n_layers=2)
    assert torch.equal(s.bounds[1], other[1])
    assert (s.bounds[0] == 0).sum() == (other[1] != 7).sum()    # (layer 0 holds nothing but NaN)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bounds_of_what_is_not_finite(dtype):
    s = Long(dtype, [130, 64], [1, 1], 4, 2, 64, 32, 16)
    s.put(0, 3, NAN, "k")
    s.put(0, 17, math.inf, "k")
    s.put(0, 40, -math.inf, "k")
    for i in range(16):
        s.put(0, 64 + i, NAN, "k")
        s.put(0, 80 + i, -math.inf, "k")
        s.put(1, 16 + i, math.inf, "k")
    s.update()
    assert torch.equal(s.bounds.double().cpu(), s.want_bounds())
    assert (s.select(3, 0, 0).cpu().numpy() == s.want_choice(3, 0, 0)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_choice_and_attention(case, dtype):
    lens, rows, hq, hkv, d, page, block, slot_major = CASES[case]
    s = Long(dtype, lens, rows, hq, hkv, d, page, block, slot_major, seed=case)
    s.update()
    for n_select, sinks, recent in CHOICES:
        blocks = s.select(n_select, sinks, recent)
        assert (blocks.cpu().numpy() == s.want_choice(n_select, sinks, recent)).all()
        out = s.attend(blocks, sinks, recent)
        s.check_attention(out, blocks.cpu(), sinks, recent)
    # all blocks: the attention over everything
    full = s.select(4096, 0, 0)
    s.check(s.attend(full, 0, 0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("absent", [False, True])
def test_trees(absent, dtype):
    rng = np.random.default_rng(2)
    rows = [8, 1, 64, 0, 33]
    s = Long(dtype, [700, 31, 260, 5, 4], rows, 8, 2, 64, 32, 16, True)
    s.update()
    for n_select, sinks, recent in CHOICES[:4]:
        par = [random_tree(rng, n, absent=absent) for n in rows]
        blocks = s.select(n_select, sinks, recent)
        assert (blocks.cpu().numpy() == s.want_choice(n_select, sinks, recent)).all()
        out = s.attend(blocks, sinks, recent, par)
        s.check_attention(out, blocks.cpu(), sinks, recent, par)
        at = 0
        for p in par:                                          # a row that is no node gets zeros
            for t, a in enumerate(O.ancestors(p)):
                if a is None:
                    assert not out[at + t].any()
            at += len(p)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ties_and_queries_that_are_not_finite(dtype):
    s = Long(dtype, [1600], [4], 6, 2, 128, 16, 16)
    for pos in range(80, 1600):                                # five blocks, over and over
        b = pos // 16 % 5
        s.cache.k[s.layer, int(s.table[s.seqs[0], pos // 16]), :, pos % 16] = s.cache.k[s.layer, int(s.table[s.seqs[0], b]), :, pos % 16]
        s.k[0][pos] = s.k[0][16 * b + pos % 16]
    s.q[1] = 0.0                                               # every block ties
    s.q[2, 0], s.q[2, 1] = NAN, math.inf
    s.q[3] = NAN
    s.q64 = s.q.double().numpy()
    s.update()
    for n_select in (1, 7, 20, 33, 64, 99):
        blocks = s.select(n_select, 16, 0)
        assert (blocks.cpu().numpy() == s.want_choice(n_select, 16, 0)).all()
        assert blocks[1, 0].tolist() == blocks[3, 1].tolist() == list(range(1, n_select + 1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lists_of_a_callers_own_making(dtype):
    s = Long(dtype, [400, 90], [2, 1], 8, 2, 128, 16, 16)      # blocks 1 .. 23 of entry 0, 1 .. 3 of entry 1 (sinks 5, recent 20)
    lists = [[2, 2, 9, 8, 23, 24, 1000], [-5, -1, 0, 3, 3, 3, 22], [1, 3, 4, 4, 5, 5, 5]]
    counts = [[2, 9, 23], [3, 22], [1, 3]]                     # not above the one before, outside, or behind the third of three
    blocks = ints([[x, x] for x in lists]).contiguous()
    want = torch.full((3, 2, 3), -1)
    for r, c in enumerate(counts):
        want[r, :, :len(c)] = torch.tensor(c)
    s.check_attention(s.attend(blocks, 5, 20), want, 5, 20)
    # numbers far out of range
    wild = torch.full((3, 2, 9), 0x7fffffff, dtype=torch.int32, device="cuda")
    wild[:, :, 0] = -0x80000000
    s.check_attention(s.attend(wild, 5, 20), torch.full((3, 2, 1), -1), 5, 20)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [NAN, math.inf, -math.inf])
def test_what_a_row_does_not_read_does_not_matter(dtype, bad):
    s = Long(dtype, [300, 90], [4, 3], 8, 2, 128, 16, 16)
    s.update()
    blocks = s.select(4, 3, 20)
    read = {(e, b) for e, lo, hi in ((0, 0, 4), (1, 4, 7)) for b in blocks[lo:hi].flatten().tolist() if b >= 0}
    for e, n in ((0, 300), (1, 90)):
        front, tail = O.block_parts(n, 16, 16, 3, 20)
        for b in range(front // 16, tail // 16):
            if (e, b) not in read:
                s.put(e, b * 16 + 5, bad)
    s.check_attention(s.attend(blocks, 3, 20), blocks.cpu(), 3, 20)
    # a late row's own value: the rows before it are as they were, the row's channel is not
    s.put(0, 302, bad, "v")
    out = s.attend(blocks, 3, 20)
    assert torch.isfinite(out[[0, 1, 4, 5, 6]].float()).all() and not torch.isfinite(out[2:4].float()).any()
    # one channel of a sink: of all rows, and of no other channel
    s.put(0, 302, 0.5, "v")
    s.cache.v[s.layer, int(s.table[s.seqs[0], 0]), :, 1, 77] = bad
    out = s.attend(blocks, 3, 20).float()
    assert torch.isfinite(out[:4, :, :77]).all() and torch.isfinite(out[:4, :, 78:]).all()
    same = out[:4, :, 77].isnan() if math.isnan(bad) else out[:4, :, 77] == bad
    assert same.all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bounds_on_lengths_and_sequences_that_are_none(dtype):
    import paper_2412_01380_amd as D
    s = Long(dtype, [300, 90], [3, 2], 8, 2, 64, 16, 16)
    s.update()
    short = D.Batch(s.batch.row_start, 5, 3, seqs=s.batch.seqs, max_len=200)      # of entry 0 the first 200 positions
    s.batch = short
    blocks = s.select(5, 1, 10)
    front, tail = O.block_parts(200, 16, 16, 1, 10)
    assert (blocks[:3] < tail // 16).all()
    s.check_attention(s.attend(blocks, 1, 10), blocks.cpu(), 1, 10, max_len=200)
    s = Long(dtype, [300, 90], [3, 2], 8, 2, 64, 16, 16)
    s.batch.seqs[0] = -4
    s.update()
    blocks = s.select(5, 1, 10)
    out = s.attend(blocks, 1, 10)
    assert (blocks[:3] == -1).all() and not out[:3].any() and torch.isfinite(out[3:].float()).all()
    # rows behind the last sequence are left as they were, and no more than max_rows of an entry are looked at
    b = D.Batch(ints([0, 3, 5]), 7, 2, seqs=ints([s.seqs[0], s.seqs[1]]))
    q = torch.zeros(7, 8, 64, dtype=DT[dtype], device="cuda")
    out = torch.full_like(q, 5.0)
    blocks = torch.full((7, 2, 3), -9, dtype=torch.int32, device="cuda")
    D.dip_select_blocks(s.cache, s.layer, b, q, s.bounds, 1, 10, blocks, workspace(D.dip_select_blocks_workspace_bytes(s.cache, b, 8, 16)))
    assert (blocks[[2, 5, 6]] == -9).all() and (blocks[[0, 1, 3, 4]] != -9).all()
    s.attend(blocks, 1, 10, q=q, out=out, batch=b)
    assert (out[[2, 5, 6]] == 5.0).all() and (out[[0, 1, 3, 4]] != 5.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_rows(dtype):
    s = Long(dtype, [300, 90], [3, 2], 8, 2, 64, 16, 16)
    s.update()
    wide = torch.full((5, 20, 64), NAN, dtype=DT[dtype], device="cuda")
    wide[:, 3:11] = s.q.cuda()
    blocks = s.select(5, 1, 10)
    assert torch.equal(s.select(5, 1, 10, q=wide[:, 3:11]), blocks)
    out = wide[:, 12:]
    assert torch.equal(s.attend(blocks, 1, 10, q=wide[:, 3:11], out=out), s.attend(blocks, 1, 10))
    assert wide[:, :3].isnan().all() and wide[:, 11].isnan().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_same_bits_every_time_and_in_graphs(dtype):
    import paper_2412_01380_amd as D
    s = Long(dtype, [3000, 900, 64], [1, 1, 1], 8, 2, 128, 16, 16)
    s.update()
    q, blocks = s.q.cuda(), torch.empty(3, 2, 20, dtype=torch.int32, device="cuda")
    ws = workspace(max(D.dip_select_blocks_workspace_bytes(s.cache, s.batch, 8, 16),
                       D.dip_block_attention_workspace_bytes(s.cache, s.batch, 8, 16, 20, 4, 50)))
    outs, graphs = [torch.empty_like(q) for _ in range(2)], [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph, out in zip(graphs, outs):                       # two graphs that share a workspace
        with torch.cuda.graph(graph):
            D.dip_kv_block_bounds(s.cache, s.layer, 1, s.seqs_dev, 0, s.bounds)
            D.dip_select_blocks(s.cache, s.layer, s.batch, q, s.bounds, 4, 50, blocks, ws)
            D.dip_block_attention(s.cache, s.layer, s.batch, None, blocks, 16, q, 0.1, 4, 50, out, ws)
    for i in range(4):
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(i)))
        s.cache.seq_len[torch.tensor(s.seqs, device="cuda")] = ints([3000 - 700 * i, 900 - 250 * i, 64 - 20 * i])
        want_blocks = s.select(20, 4, 50, q=q)
        want = torch.empty_like(q)
        D.dip_block_attention(s.cache, s.layer, s.batch, None, want_blocks, 16, q, 0.1, 4, 50, want, ws)
        for graph, out in zip(graphs, outs):
            out.fill_(NAN), blocks.fill_(-9)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want) and torch.equal(blocks, want_blocks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_closer_than_fp32_tells(dtype):
    # blocks whose scores differ by less than fp32 sums do: the order of the 64-bit sums decides
    s = Long(dtype, [3200], [3], 4, 2, 128, 16, 16, wide=1.0)
    base = s.cache.k[s.layer, int(s.table[s.seqs[0], 0])].clone()
    g = torch.Generator().manual_seed(1)
    for j in range(200):
        page = base.clone()
        at = torch.randint(0, 128, (4,), generator=g).cuda()
        page[..., at] *= 1 + (0.0078125 if dtype == "bf16" else 2.0 ** -20) * (j % 7)
        s.cache.k[s.layer, int(s.table[s.seqs[0], j])] = page
        s.k[0][j * 16:(j + 1) * 16] = page.transpose(0, 1).double().cpu().numpy()
    s.q[1] *= 1e-3
    s.q64 = s.q.double().numpy()
    s.update()
    for n_select in (1, 13, 50, 128, 199):
        assert (s.select(n_select, 0, 0).cpu().numpy() == s.want_choice(n_select, 0, 0)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_blocks(dtype):
    # more than a workgroup holds at a time, and rows of very different sizes beside each other
    s = Long(dtype, [80000], [2], 2, 1, 64, 16, 16, seed=4)
    s.q[0] *= 1e4
    s.q64 = s.q.double().numpy()
    s.update()
    for n_select in (1, 700, 4096):
        blocks = s.select(n_select, 5, 1000)
        assert (blocks.cpu().numpy() == s.want_choice(n_select, 5, 1000)).all()
