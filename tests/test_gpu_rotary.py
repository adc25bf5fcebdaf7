"""Rows turned to their positions, alone and on their way into a paged cache, against the 64-bit oracle: layouts, parts of
heads of any even size, far and negative positions, strides, trees, pages that are another's."""
import math

import numpy as np
import pytest
import torch

from oracle import decode_oracle as O
from test_gpu_decode import DT, NAN, ints, random_tree, starts

pytestmark = pytest.mark.gpu


def bound(x, positions, freq, ref, dtype, scale=1.0):
    """What the turned rows may be off by: the reduced angle is rounded to fp32 (1.6 units of 2^-24), sine and cosine are off
    by up to 4 units in the last place (8), their scale, two products and a sum are rounded (4), all of |a| + |b|; the angle
    itself is a product of three fp64 numbers.  bf16 outputs are rounded by up to 2^-8."""
    half = len(freq)
    mag = np.abs(x).max(-1, keepdims=True) * 2 * abs(scale)
    far = np.abs(np.asarray(positions, dtype=np.float64))[:, None, None] * np.max(freq) * 2.0 ** -51
    out = mag * (14 * 2.0 ** -24 + far) + 1e-37
    return out + (np.abs(ref) * 2.0 ** -8 if dtype == "bf16" else 0) if half else out


def rotaries(D, dims, scale=1.0):
    f = D.dip_rotary_frequencies(dims)
    return f.numpy(), {lay: D.Rotary(f.cuda(), lay, scale) for lay in (D.DIP_ROTARY_HALF, D.DIP_ROTARY_INTERLEAVED)}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,heads,dim,dims", [(1, 1, 64, 64), (7, 32, 96, 96), (3, 5, 128, 2), (33, 3, 128, 32), (5, 2, 96, 24),
                                                 (9, 4, 128, 126), (2, 3, 64, 50), (40, 7, 128, 72), (3, 2, 1024, 1024), (2, 1, 4608, 4096),
                                                 (1500, 2, 64, 20), (5000, 1, 128, 128)])
def test_rows(rows, heads, dim, dims, dtype):
    import paper_2412_01380_amd as D
    g = torch.Generator().manual_seed(rows)
    x = torch.randn(rows, heads, dim, generator=g).to(DT[dtype])
    pos = torch.randint(0, 100000, (rows,), generator=g).tolist()
    pos[:4] = [0, -3, 1 << 20, (1 << 31) - 1][:rows]
    freq, rot = rotaries(D, dims)
    for lay, r in rot.items():
        out = torch.full_like(x, NAN, device="cuda")
        D.dip_rotate_rows(r, x.cuda(), ints(pos), out)
        ref = O.turn(x.double().numpy(), pos, freq, lay == D.DIP_ROTARY_INTERLEAVED)
        err = np.abs(out.double().cpu().numpy() - ref)
        assert (err <= bound(x.double().numpy(), pos, freq, ref, dtype)).all()
        assert torch.equal(out[:, :, dims:].cpu(), x[:, :, dims:])             # what is not turned keeps its bits
        again = x.cuda()
        D.dip_rotate_rows(r, again, ints(pos), again)                          # in place: the same bits
        assert torch.equal(again, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_rows_leave_their_neighbours_alone(dtype):
    import paper_2412_01380_amd as D
    g = torch.Generator().manual_seed(1)
    wide = torch.randn(19, 11, 64, generator=g).to(DT[dtype]).cuda()
    before = wide.clone()
    freq, rot = rotaries(D, 48, 1.25)
    pos = list(range(100, 119))
    for lay, r in rot.items():
        wide.copy_(before)
        # columns of one array: heads 2 .. 4 turned into heads 6 .. 8
        D.dip_rotate_rows(r, wide[:, 2:5], ints(pos), wide[:, 6:9])
        x = before[:, 2:5].double().cpu().numpy()
        ref = O.turn(x, pos, freq, lay == D.DIP_ROTARY_INTERLEAVED, 1.25)
        assert (np.abs(wide[:, 6:9].double().cpu().numpy() - ref) <= bound(x, pos, freq, ref, dtype, 1.25)).all()
        assert torch.equal(wide[:, :6], before[:, :6]) and torch.equal(wide[:, 9:], before[:, 9:])
        with pytest.raises(D.DipError):
            D.dip_rotate_rows(r, wide[:, 2:5], ints(pos), wide[:, 4:7])


class Step:
    """Rows of a step for sequences of given lengths, in a cache full of NaN whose pages are shuffled and whose own."""

    def __init__(self, dtype, lens, rows, hq, hkv, d, page, slot_major=False, seed=0, layers=2, no_room=(), parents=None):
        import paper_2412_01380_amd as D
        g = torch.Generator().manual_seed(seed)
        dt = DT[dtype]
        self.lens, self.rows, self.dtype, self.page, self.parents = lens, rows, dtype, page, parents
        need = [-(-(n + r) // page) for n, r in zip(lens, rows)]
        n_pages, max_pages = sum(need) + 2, max(need) + 1
        order = torch.randperm(n_pages, generator=g).tolist()
        self.seqs = torch.randperm(len(lens) + 1, generator=g)[:len(lens)].tolist()
        self.table = torch.full((len(lens) + 1, max_pages), -1, dtype=torch.int32)
        seq_len, refs, at = torch.zeros(len(lens) + 1, dtype=torch.int32), torch.zeros(n_pages, dtype=torch.int32), 0
        for i, (s, n, m) in enumerate(zip(self.seqs, lens, need)):
            self.table[s, :m] = torch.tensor(order[at:at + m], dtype=torch.int32)
            refs[order[at:at + m]] = 1
            if i in no_room:
                refs[order[at + m - 1]] = 2
            at, seq_len[s] = at + m, n
        shape = (layers, n_pages, page, hkv, d) if slot_major else (layers, n_pages, hkv, page, d)
        k, v = (torch.full(shape, NAN, dtype=dt, device="cuda") for _ in range(2))
        k, v = (k.transpose(2, 3), v.transpose(2, 3)) if slot_major else (k, v)
        self.cache = D.KvCache(k, v, self.table.cuda(), seq_len.cuda(), refs.cuda())
        self.n = sum(rows)
        self.fused = torch.randn(self.n, hq + 2 * hkv, d, generator=g).to(dt).cuda()
        self.q, self.k, self.v = self.fused.split([hq, hkv, hkv], 1)
        self.batch = D.Batch(starts(rows), self.n, max(rows), seqs=ints(self.seqs))
        self.pos = []
        for i, (n, r) in enumerate(zip(lens, rows)):
            self.pos += O.tree_positions(n, parents[i]) if parents else list(range(n, n + r))

    def run(self, rot, layer, q_out, q=None, k=None, v=None):
        import paper_2412_01380_amd as D
        par = ints([x for p in self.parents for x in p]) if self.parents else None
        D.dip_kv_append_rotary(self.cache, layer, self.batch, par, rot, self.q if q is None else q, q_out, self.k if k is None else k,
                               self.v if v is None else v)

    def check(self, freq, inter, layer, q_out, passed_over=()):
        """Every place of the cache: the rows' own, and NaN elsewhere."""
        want_k, want_v = (torch.full(self.cache.k.shape, NAN, dtype=torch.float64) for _ in range(2))
        tol = torch.zeros(self.cache.k.shape, dtype=torch.float64)
        x = self.k.double().cpu().numpy()
        ref = O.turn(x, self.pos, freq, inter)
        off, at = bound(x, self.pos, freq, ref, self.dtype), 0
        for i, (n, r) in enumerate(zip(self.lens, self.rows)):
            for t in range(r if i not in passed_over else 0):
                pg, sl = int(self.table[self.seqs[i], (n + t) // self.page]), (n + t) % self.page
                want_k[layer, pg, :, sl], tol[layer, pg, :, sl] = torch.from_numpy(ref[at + t]), torch.from_numpy(off[at + t])
                want_v[layer, pg, :, sl] = self.v[at + t].double().cpu()
            at += r
        got = self.cache.k.double().cpu()
        assert torch.equal(got.isnan(), want_k.isnan())
        assert ((got - want_k).abs().nan_to_num(0.0) <= tol).all()
        assert torch.equal(self.cache.v.double().cpu().nan_to_num(1e9), want_v.nan_to_num(1e9))
        if q_out is not None:
            x = self.q.double().cpu().numpy()
            ref = O.turn(x, self.pos, freq, inter)
            assert (np.abs(q_out.double().cpu().numpy() - ref) <= bound(x, self.pos, freq, ref, self.dtype)).all()


APPENDS = [
    # lens, rows, hq, hkv, d, page, slot_major, dims
    ([0], [1], 1, 1, 64, 16, False, 64),
    ([700, 3], [1, 1], 32, 8, 128, 16, False, 128),
    ([15, 16, 0, 31], [3, 17, 0, 1], 6, 2, 96, 16, True, 24),
    ([100, 0], [70, 33], 10, 5, 64, 32, False, 18),
    ([5], [300], 3, 3, 128, 1, True, 96),
    ([4097, 9, 1], [600, 200, 400], 2, 1, 32, 128, False, 32),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(APPENDS)))
def test_append(case, dtype):
    import paper_2412_01380_amd as D
    lens, rows, hq, hkv, d, page, slot_major, dims = APPENDS[case]
    freq, rot = rotaries(D, dims)
    for lay, r in rot.items():
        s = Step(dtype, lens, rows, hq, hkv, d, page, slot_major, seed=case)
        out = torch.full((s.n, hq, d), NAN, dtype=DT[dtype], device="cuda")
        s.run(r, 1, out)
        s.check(freq, lay == D.DIP_ROTARY_INTERLEAVED, 1, out)
        # the keys alone; queries in place; the same bits
        twin = Step(dtype, lens, rows, hq, hkv, d, page, slot_major, seed=case)
        D.dip_kv_append_rotary(twin.cache, 1, twin.batch, None, r, None, None, twin.k, twin.v)
        same = lambda a, b: torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0))
        assert same(twin.cache.k, s.cache.k) and same(twin.cache.v, s.cache.v)
        twin.run(r, 1, twin.q)
        assert torch.equal(twin.q, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_trees(dtype):
    import paper_2412_01380_amd as D
    rng = np.random.default_rng(5)
    rows = [64, 1, 0, 9, 33]
    par = [random_tree(rng, n, absent=i % 2 == 0) for i, n in enumerate(rows)]
    freq, rot = rotaries(D, 64)
    for lay, r in rot.items():
        s = Step(dtype, [30, 0, 5, 100, 7], rows, 8, 2, 64, 16, parents=par)
        out = torch.full((s.n, 8, 64), NAN, dtype=DT[dtype], device="cuda")
        s.run(r, 0, out)
        s.check(freq, lay == D.DIP_ROTARY_INTERLEAVED, 0, out)


def test_entries_without_room_are_passed_over():
    import paper_2412_01380_amd as D
    freq, rot = rotaries(D, 64)
    s = Step("bf16", [20, 5, 40], [4, 3, 30], 4, 2, 64, 16, no_room=(1,))
    out = torch.full((s.n, 4, 64), NAN, dtype=torch.bfloat16, device="cuda")
    s.run(rot[0], 1, out)
    s.check(freq, False, 1, out, passed_over=(1,))             # its queries are turned all the same
    # a table that ends before the rows do, and a sequence that is none
    s = Step("f32", [20, 5], [4, 3], 4, 2, 64, 16)
    s.cache.page_table[s.seqs[0], 1] = -1
    out = torch.full((s.n, 4, 64), NAN, dtype=torch.float32, device="cuda")
    s.run(rot[0], 0, out)
    s.check(freq, False, 0, out, passed_over=(0,))
    s = Step("f32", [20, 5], [4, 3], 4, 2, 64, 16)
    s.batch.seqs[0] = 77
    out = torch.full((s.n, 4, 64), NAN, dtype=torch.float32, device="cuda")
    s.run(rot[0], 0, out)
    assert out[:4].isnan().all() and not out[4:].isnan().any()
    s.check(freq, False, 0, None, passed_over=(0,))


def test_a_graph_follows_lengths_and_rows():
    import paper_2412_01380_amd as D
    freq, rot = rotaries(D, 64)
    s = Step("f32", [20, 5], [4, 3], 4, 2, 64, 16)
    out = torch.empty(s.n, 4, 64, device="cuda")
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s.run(rot[0], 0, out)
    for i in range(3):
        s.fused.copy_(torch.randn(s.fused.shape, generator=torch.Generator().manual_seed(i)))
        s.cache.k.fill_(NAN), s.cache.v.fill_(NAN)
        lens = [20 + i, 5 + i]
        s.cache.seq_len[torch.tensor(s.seqs, device="cuda")] = ints(lens)
        s.lens, s.pos = lens, [p for n, r in zip(lens, s.rows) for p in range(n, n + r)]
        graph.replay()
        torch.cuda.synchronize()
        s.check(freq, False, 0, out)
