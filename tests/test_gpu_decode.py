"""Attention over a paged cache, verification of drafted trees and page operations against the 64-bit
oracle: head layouts, page sizes, lengths from nothing to long, odd sizes, strides, masks that leave a row
empty, and whatever lies in places that nobody sees."""
import math

import numpy as np
import pytest
import torch

from oracle import decode_oracle as O

pytestmark = pytest.mark.gpu

NAN = float("nan")
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def starts(rows):
    return ints([0] + list(np.cumsum(rows)))


def workspace(n):
    # (filled with what would show as NaN or a wrong count if it were read before it is written)
    return torch.full((max(n, 256),), 0xff, dtype=torch.uint8, device="cuda")


class Setup:
    """Sequences of given lengths with rows on top of them in a cache of shuffled pages; everything that is
    no sequence's position holds NaN."""

    def __init__(self, dtype, lens, rows, hq, hkv, d, page, slot_major=False, seed=0, layers=2, layer=1, spare=3, wide=1.0):
        import paper_2412_01380_amd as D
        g = torch.Generator().manual_seed(seed)
        dt = DT[dtype]
        self.lens, self.rows, self.hq, self.hkv, self.d, self.layer, self.dtype = lens, rows, hq, hkv, d, layer, dtype
        need = [-(-(n + r) // page) for n, r in zip(lens, rows)]
        n_pages, self.max_pages = sum(need) + spare, max(max(need), 1) + 1
        order = torch.randperm(n_pages, generator=g).tolist()
        table = torch.full((len(lens) + 1, self.max_pages), -1, dtype=torch.int32)
        self.seqs = torch.randperm(len(lens) + 1, generator=g)[:len(lens)].tolist()
        shape = (layers, n_pages, page, hkv, d) if slot_major else (layers, n_pages, hkv, page, d)
        k, v = torch.full(shape, NAN, dtype=dt), torch.full(shape, NAN, dtype=dt)
        k, v = (k.transpose(2, 3), v.transpose(2, 3)) if slot_major else (k, v)
        seq_len = torch.zeros(len(lens) + 1, dtype=torch.int32)
        self.k, self.v, at = [], [], 0
        for s, n, r, m in zip(self.seqs, lens, rows, need):
            table[s, :m] = torch.tensor(order[at:at + m], dtype=torch.int32)
            at += m
            seq_len[s] = n
            kk = (wide * torch.randn(n + r, hkv, d, generator=g)).to(dt)
            vv = torch.randn(n + r, hkv, d, generator=g).to(dt)
            pos = torch.arange(n + r)
            pg, sl = table[s][pos // page].long(), pos % page
            k[layer, pg, :, sl], v[layer, pg, :, sl] = kk, vv
            self.k.append(kk.double().numpy())
            self.v.append(vv.double().numpy())
        n_rows = sum(rows)
        self.q = torch.randn(n_rows, hq, d, generator=g).to(dt)
        self.q64 = self.q.double().numpy()
        refs = torch.zeros(n_pages, dtype=torch.int32)
        dev = lambda t: t.transpose(2, 3).contiguous().cuda().transpose(2, 3) if slot_major and t.dim() == 5 else t.cuda()
        self.table = table
        self.cache = D.KvCache(dev(k), dev(v), dev(table), dev(seq_len), dev(refs))
        self.batch = D.Batch(starts(rows), n_rows, max(rows), seqs=ints(self.seqs), max_len=max(n + r for n, r in zip(lens, rows)))

    def put(self, entry, pos, value, which="kv"):
        """Overwrite one position of an entry's sequence (on the device and for the oracle)."""
        page = self.cache.k.shape[3]
        pg, sl = int(self.table[self.seqs[entry], pos // page]), pos % page
        for name in which:
            getattr(self.cache, name)[self.layer, pg, :, sl] = value
            getattr(self, name)[entry][pos] = value

    def run(self, window=0, sinks=0, parents=None, q=None, out=None, batch=None, ws=None, stream=None):
        import paper_2412_01380_amd as D
        q = self.q.cuda() if q is None else q
        out = torch.full((len(q), self.hq, self.d), NAN, dtype=q.dtype, device="cuda") if out is None else out
        b = batch or self.batch
        ws = workspace(D.dip_attention_workspace_bytes(self.cache, b, self.hq, window, sinks)) if ws is None else ws
        scale = 1 / math.sqrt(self.d)
        if parents is None:
            D.dip_window_attention(self.cache, self.layer, b, q, scale, window, sinks, out, ws, stream)
        else:
            D.dip_tree_attention(self.cache, self.layer, b, ints([x for p in parents for x in p]), q, scale, window, sinks, out, ws, stream)
        return out

    def check(self, out, window=0, sinks=0, parents=None):
        """Every element within the rounding of the definition: scores are fp32 sums of d products, weights are
        exponentials of them, the sums over the keys are fp32, and with bf16 the weights and the output are
        rounded to 8 bits."""
        got, at = out.double().cpu().numpy(), 0
        for i, (n, r) in enumerate(zip(self.lens, self.rows)):
            sees = O.visible(n, r, window, sinks, None if parents is None else parents[i])
            # (what nobody sees may be anything; the oracle must not multiply it by nothing)
            ref, mag, big = O.attend(self.q64[at:at + r], self.k[i], self.v[i], sees, 1 / math.sqrt(self.d))
            keys = n + r
            dz = (big * (self.d / 4 + 8) + 64)[..., None] * 2.0 ** -24
            bound = mag * (2 * dz + (4 * math.sqrt(keys) + 32) * 2.0 ** -24) + 1e-30
            if self.dtype == "bf16":
                bound = bound + (mag + np.abs(ref)) * 2.0 ** -8.9
            err = np.abs(got[at:at + r] - ref)
            assert np.isfinite(got[at:at + r]).all(), ("not finite", i)
            assert (err <= bound).all(), (i, float((err / bound).max()))
            at += r


CASES = [
    # lens, rows, hq, hkv, d, page, slot_major
    ([0], [1], 1, 1, 64, 16, False),                       # the first token of all
    ([0, 5, 1], [1, 1, 1], 4, 2, 128, 16, True),
    ([31, 32, 33, 63, 64, 65], [1] * 6, 8, 8, 96, 8, False),
    ([700, 3, 129], [1, 1, 1], 32, 4, 128, 16, False),     # eight query heads share one
    ([511, 0, 40], [3, 70, 0], 10, 2, 64, 32, True),       # an entry without rows
    ([100, 17], [129, 33], 6, 3, 128, 64, False),
    ([1, 257], [40, 31], 7, 1, 96, 1, True),               # pages of one slot
    ([2500, 33], [2, 1], 5, 5, 64, 128, False),            # long enough for shares
    ([20], [300], 8, 1, 128, 16, True),
]
MASKS = [(0, 0), (1, 0), (7, 0), (64, 4), (100, 33), (0x7fffffff, 5)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_window_attention(case, dtype):
    lens, rows, hq, hkv, d, page, slot_major = case
    s = Setup(dtype, lens, rows, hq, hkv, d, page, slot_major, seed=len(rows))
    for window, sinks in MASKS:
        s.check(s.run(window, sinks), window, sinks)


def random_tree(rng, n, kids=3, absent=False):
    par = [-1] if n else []
    for t in range(1, n):
        up = int(rng.integers(max(0, t - kids), t))
        par.append(up)
    if absent and n > 2:
        for t in rng.choice(np.arange(1, n), size=max(1, n // 5), replace=False):
            par[t] = int(rng.choice([-2, -77, t, t + 3, 1000]))
    return par


TREES = [
    ([0], [1], 1, 1, 64, 16, False),
    ([9, 0], [7, 5], 4, 4, 96, 32, True),
    ([1000, 31, 5], [8, 1, 3], 32, 8, 128, 16, False),
    ([333, 64], [64, 63], 10, 2, 128, 64, False),
    ([4100, 12], [33, 20], 8, 1, 64, 8, True),
    ([70, 3], [16, 9], 14, 2, 96, 128, False),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("absent", [False, True])
@pytest.mark.parametrize("case", TREES, ids=[str(i) for i in range(len(TREES))])
def test_tree_attention(case, absent, dtype):
    lens, rows, hq, hkv, d, page, slot_major = case
    s = Setup(dtype, lens, rows, hq, hkv, d, page, slot_major, seed=7)
    rng = np.random.default_rng(3)
    for window, sinks in [(0, 0), (1, 0), (40, 3), (500, 0)]:
        par = [random_tree(rng, n, absent=absent) for n in rows]
        out = s.run(window, sinks, par)
        s.check(out, window, sinks, par)
        at = 0
        for p in par:                                      # a row that is no node gets zeros
            for t, a in enumerate(O.ancestors(p)):
                if a is None:
                    assert not out[at + t].any()
            at += len(p)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [NAN, math.inf, -math.inf])
def test_what_a_row_does_not_see_does_not_matter(dtype, bad):
    # positions in front of the window, behind a row, and a sibling's
    s = Setup(dtype, [300, 90], [40, 20], 8, 2, 128, 16)
    for e, pos in [(0, 7), (0, 200), (1, 4), (1, 30)]:     # sinks 3, window 64: row 0 sees from 237 and from 27
        if pos + 64 <= [300, 90][e]:
            s.put(e, pos, bad)
    s.check(s.run(64, 3), 64, 3)
    # a late row's own position: the rows before it do not see it, the row itself does
    s.put(0, 339, bad)
    out = s.run(64, 3)
    rest = [r for r in range(60) if r != 39]
    assert torch.isfinite(out[rest].float()).all() and not torch.isfinite(out[39].float()).all()
    # trees: a sibling that is not finite
    s = Setup(dtype, [50], [8], 4, 1, 64, 32)
    par = [-1, 0, 0, 1, 1, 2, 3, 5]
    s.put(0, 52, bad)                                      # node 2, seen by 2, 5, 7
    out = s.run(0, 0, [par])
    clean = Setup(dtype, [50], [8], 4, 1, 64, 32).run(0, 0, [par])
    for t in range(8):
        if t in (2, 5, 7):
            assert not torch.isfinite(out[t].float()).all()
        else:
            assert torch.equal(out[t], clean[t])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores_and_equal_scores(dtype):
    s = Setup(dtype, [400], [5], 4, 2, 128, 16, wide=30.0)     # scores in the hundreds: nearly one key decides
    got = s.run(128, 2).double().cpu().numpy()
    ref, mag, _ = O.attend(s.q64, s.k[0], s.v[0], O.visible(400, 5, 128, 2), 1 / math.sqrt(128))
    # a score z off by z 2^-18 moves a weight by that share
    assert np.abs(got - ref).max() <= (0.02 if dtype == "bf16" else 2e-2 * 0.05) * np.abs(ref).max() + 1e-3
    z = Setup(dtype, [77], [3], 4, 2, 64, 16)
    z.q = torch.zeros_like(z.q)
    z.q64 = z.q64 * 0
    z.check(z.run(), 0, 0)                                     # the plain mean


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_rows_and_outputs(dtype):
    s = Setup(dtype, [50, 200], [4, 7], 8, 2, 128, 16)
    fused = torch.full((11, (8 + 2 + 2) * 128), NAN, dtype=DT[dtype], device="cuda")
    fused[:, :8 * 128] = s.q.cuda().view(11, -1)
    wide = torch.full((11, 9, 128), 3.0, dtype=DT[dtype], device="cuda")
    out = s.run(32, 1, q=fused[:, :8 * 128].unflatten(1, (8, 128)), out=wide[:, :8])
    s.check(out, 32, 1)
    assert (wide[:, 8] == 3.0).all()


def test_same_bits_every_time_and_on_another_stream():
    s = Setup("bf16", [5000, 200], [8, 5], 32, 8, 128, 16)
    par = [random_tree(np.random.default_rng(1), n) for n in s.rows]
    first = s.run(0, 0, par)
    for _ in range(5):
        assert torch.equal(s.run(0, 0, par), first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = s.run(0, 0, par, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, first)


def test_offsets_beyond_32_bits():
    import paper_2412_01380_amd as D
    page, hkv, d = 64, 8, 128
    n_pages = (1 << 32) // (page * hkv * d) + 40               # over 2^32 elements of k, and of v
    k = torch.empty(1, n_pages, hkv, page, d, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    n, r = 300, 3
    used = list(range(n_pages - 5, n_pages))
    g = torch.Generator().manual_seed(5)
    kk, vv = (torch.randn(n + r, hkv, d, generator=g).bfloat16() for _ in range(2))
    q = torch.randn(r, 16, d, generator=g).bfloat16()
    table = ints([used])
    seq_len, refs = ints([0]), torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    refs[used] = 1
    cache = D.KvCache(k, v, table, seq_len, refs)
    all_rows = D.Batch(ints([0, n + r]), n + r, n + r, seqs=ints([0]))
    D.dip_kv_append(cache, 0, all_rows, kk.cuda(), vv.cuda())
    seq_len.fill_(n)
    b = D.Batch(ints([0, r]), r, r, seqs=ints([0]), max_len=n + r)
    out = torch.empty(r, 16, d, dtype=torch.bfloat16, device="cuda")
    ws = workspace(D.dip_attention_workspace_bytes(cache, b, 16))
    D.dip_window_attention(cache, 0, b, q.cuda(), d ** -0.5, 0, 0, out, ws)
    ref, mag, _ = O.attend(q.double().numpy(), kk.double().numpy(), vv.double().numpy(), O.visible(n, r, 0, 0), d ** -0.5)
    assert np.abs(out.double().cpu().numpy() - ref).max() <= 2.0 ** -8 * mag.max() + 1e-4


def test_lengths_and_tables_out_of_range_stay_in_bounds():
    # a table full of nonsense, lengths beyond the table, sequences that do not exist, rows beyond the bounds:
    # results are unspecified, other entries' are right
    s = Setup("bf16", [200, 60, 90], [2, 3, 1], 8, 2, 128, 16)
    good = s.run(0, 0)
    s.cache.page_table[s.seqs[1]] = torch.randint(-2 ** 31, 2 ** 31 - 1, (s.max_pages,), dtype=torch.int32).cuda()
    s.cache.seq_len[s.seqs[2]] = 2 ** 31 - 1
    out = s.run(0, 0)
    assert torch.equal(out[:2], good[:2])
    s.batch.seqs[1] = 10 ** 6
    s.cache.seq_len[s.seqs[2]] = -5
    assert torch.equal(s.run(0, 0)[:2], good[:2])
    s.batch.row_start[3] = 2 ** 30
    assert torch.equal(s.run(0, 0)[:2], good[:2])


def test_attention_in_a_graph_follows_the_lengths():
    s = Setup("bf16", [900, 20], [1, 1], 8, 2, 128, 16)
    ws = workspace(1 << 22)
    q, out = s.q.cuda(), torch.empty(2, 8, 128, dtype=torch.bfloat16, device="cuda")
    s.run(256, 4, q=q, out=out, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run(256, 4, q=q, out=out, ws=ws)
    for n in (900, 17, 500, 899, 1):
        s.cache.seq_len[s.seqs[0]] = n
        out.fill_(NAN)
        eager = s.run(256, 4, q=q).clone()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


# ---- verification --------------------------------------------------------------------------------------------
def verify_inputs(rng, trees, vocab, sharp=2.0, near=0.5, dtype=torch.float32):
    n = sum(len(t) for t in trees)
    logits = rng.normal(size=(n, vocab)) * sharp
    other = logits + near * rng.normal(size=(n, vocab))
    soft = lambda z: torch.softmax(torch.from_numpy(z), -1).to(dtype)
    p, q = soft(logits), soft(other)
    tokens, at = [], 0
    for t in trees:
        for node, up in enumerate(t):
            row = q[at + (up if 0 <= up < node else 0)].double().numpy()
            tokens.append(int(rng.choice(vocab, p=row / row.sum())))
        at += len(t)
    return p, q, tokens, rng.random(n).astype(np.float32), rng.random(len(trees)).astype(np.float32)


def run_verify(trees, p, q, tokens, u, us, kids):
    import paper_2412_01380_amd as D
    rows = [len(t) for t in trees]
    n = sum(rows)
    b = D.Batch(starts(rows), n, max(rows))
    keep, path, token = (torch.full((m,), -9, dtype=torch.int32, device="cuda") for m in (len(rows), n, len(rows)))
    ws = workspace(D.dip_verify_tree_workspace_bytes(b, p.shape[1], kids))
    D.dip_verify_tree(b, ints(tokens), ints([x for t in trees for x in t]), p.cuda() if not p.is_cuda else p,
                      q.cuda() if not q.is_cuda else q, torch.from_numpy(u).cuda(), torch.from_numpy(us).cuda(), kids, keep, path,
                      token, ws)
    return keep.tolist(), path.tolist(), token.tolist()


def check_verify(trees, p, q, tokens, u, us, kids):
    keep, path, token = run_verify(trees, p, q, tokens, u, us, kids)
    pd, qd, at = p.double().cpu().numpy(), q.double().cpu().numpy(), 0
    for i, t in enumerate(trees):
        r = slice(at, at + len(t))
        ref, tok = O.verify(t, tokens[r], pd[r], qd[r], u[r], us[i], kids)
        assert keep[i] == len(ref) and path[r] == ref + [-1] * (len(t) - len(ref)), (i, ref, path[r])
        assert token[i] == tok, (i, token[i], tok)
        at += len(t)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1, 2, 7, 100, 4096, 4097, 32064, 50257])
def test_verify_against_the_usual_rule(vocab, dtype):
    rng = np.random.default_rng(vocab)
    for kids in (1, 2, 4):
        trees = [random_tree(rng, n, kids=kids) for n in (1, 5, 16, 2, 64 if vocab < 5000 else 9)]
        check_verify(trees, *verify_inputs(rng, trees, vocab, dtype=dtype), 63)


def test_verify_stars_limits_and_absent_nodes():
    rng = np.random.default_rng(0)
    star = [-1] + [0] * 12
    for kids in (1, 3, 12, 63):
        trees = [star, [-1, 0, 0, 0, 3, 3], [0, 0], [-2, -1, 1], [-1, -1, 0, 7, 2, 3], [-1]]
        check_verify(trees, *verify_inputs(rng, trees, 500, near=3.0), kids)


def test_verify_greedy_and_degenerate_rows():
    # one-hot targets: the drafts that agree stand; identical rows: the first child always stands
    trees = [[-1, 0, 0, 1, 3], [-1, 0, 1, 2]]
    vocab = 1000
    rng = np.random.default_rng(4)
    p, q, tokens, u, us = verify_inputs(rng, trees, vocab)
    hot = torch.zeros_like(p)
    hot[torch.arange(9), torch.tensor([tokens[2], 5, 6, 7, 8, tokens[6], tokens[7], 0, 9])] = 1
    check_verify(trees, hot, q, tokens, u, us, 63)
    check_verify(trees, q, q, tokens, u, us, 63)
    check_verify(trees, hot, hot, tokens, u, us, 63)
    zero = torch.zeros_like(p)
    keep, path, token = run_verify(trees, zero, q, tokens, u, us, 63)
    assert keep == [1, 1] and token == [-1, -1]
    bad = [t if i % 2 else -5 for i, t in enumerate(tokens)]
    check_verify(trees, p, q, bad, u, us, 63)
    # the draw's ends
    for x in (0.0, float(np.nextafter(np.float32(1), np.float32(0)))):
        check_verify(trees, p, q, tokens, u, np.full(2, x, np.float32), 63)
    # nothing hangs or leaves its bounds on rows that are not finite
    nan = torch.full_like(p, NAN)
    run_verify(trees, nan, q, tokens, u, us, 63)
    run_verify(trees, p, nan, tokens, u, us, 63)


def test_verify_strided_rows():
    rng = np.random.default_rng(9)
    trees = [[-1, 0, 0, 1]]
    p, q, tokens, u, us = verify_inputs(rng, trees, 501)
    wide = torch.full((4, 777), NAN, device="cuda")
    wide[:, 3:504] = p.cuda()
    check_verify(trees, wide[:, 3:504], q, tokens, u, us, 2)


def test_verified_tokens_follow_the_target():
    # over many draws the first token behind node 0 is distributed as the target's row, whatever drafted it
    vocab, n = 6, 1024
    rng = np.random.default_rng(11)
    p = torch.tensor([[.4, .1, .2, .05, .2, .05]])
    q = torch.tensor([[.1, .3, .1, .3, .1, .1]])
    trees = [[-1, 0, 0] for _ in range(n)]
    tokens = []
    for _ in range(n):
        tokens += [0, int(rng.choice(6, p=q[0].double().numpy() / q[0].double().sum().item())),
                   int(rng.choice(6, p=q[0].double().numpy() / q[0].double().sum().item()))]
    keep, path, token = run_verify(trees, p.expand(3 * n, 6).contiguous(), q.expand(3 * n, 6).contiguous(), tokens,
                                   rng.random(3 * n).astype(np.float32), rng.random(n).astype(np.float32), 2)
    first = [tokens[3 * i + path[3 * i + 1]] if keep[i] > 1 else token[i] for i in range(n)]
    share = np.bincount(first, minlength=6) / n
    # five standard deviations of a share of 1024 draws
    assert np.all(np.abs(share - p[0].numpy()) <= 5 * np.sqrt(p[0].numpy() * (1 - p[0].numpy()) / n))


# ---- pages ---------------------------------------------------------------------------------------------------
class Paged:
    """A small cache beside the oracle's lists; a row's name is written into all of its elements."""

    def __init__(self, n_pages, page, n_seqs, max_pages, hkv=2, d=64, layers=3, dtype=torch.float32, slot_major=False):
        import paper_2412_01380_amd as D
        self.D, self.o, self.layers, self.hkv, self.d = D, O.Pool(n_pages, page, n_seqs, max_pages), layers, hkv, d
        shape = (layers, n_pages, page, hkv, d) if slot_major else (layers, n_pages, hkv, page, d)
        k, v = (torch.zeros(shape, dtype=dtype, device="cuda") for _ in range(2))
        k, v = (k.transpose(2, 3), v.transpose(2, 3)) if slot_major else (k, v)
        junk = lambda *s: torch.full(s, 77, dtype=torch.int32, device="cuda")
        self.c = D.KvCache(k, v, junk(n_seqs, max_pages), junk(n_seqs), junk(n_pages))
        D.dip_kv_init(self.c)
        self.next = 1

    def batch(self, seqs, counts):
        return self.D.Batch(starts(counts), max(1, sum(counts)), max(1, max(counts)), seqs=ints(seqs))

    def step(self, seqs, counts, paths=None, keep=None):
        b = self.batch(seqs, counts)
        granted = torch.full((len(seqs),), -1, dtype=torch.int32, device="cuda")
        ws = workspace(self.D.dip_kv_reserve_workspace_bytes(self.c, b))
        self.D.dip_kv_reserve(self.c, b, granted, ws)
        assert granted.tolist() == self.o.reserve(seqs, counts)
        self.check()
        again = granted.clone()
        self.D.dip_kv_reserve(self.c, b, again, ws)            # the same rows again: nothing changes
        if all(granted.tolist()):
            assert torch.equal(again, granted)
            self.check()
        else:
            self.o.reserve(seqs, counts)
        names = [list(range(self.next + sum(counts[:i]), self.next + sum(counts[:i + 1]))) for i in range(len(counts))]
        self.next += sum(counts)
        flat = torch.tensor([x for n in names for x in n] or [0], dtype=torch.float32, device="cuda")
        k_new = flat[None, :, None, None].expand(self.layers, -1, self.hkv, self.d).to(self.c.k.dtype)
        k_new = k_new + 1000 * torch.arange(self.layers, device="cuda")[:, None, None, None].to(k_new.dtype)
        v_new = (-k_new).contiguous()
        k_new = k_new.contiguous()
        self.D.dip_kv_append(self.c, 0, b, k_new[:1], v_new[:1])
        if self.layers > 1:
            self.D.dip_kv_append(self.c, 1, b, k_new[1:], v_new[1:])
        self.o.append(seqs, names)
        self.check()
        pt = None if paths is None else ints([x for p, n in zip(paths, counts) for x in (p + [-1] * n)[:n]] or [0])
        self.D.dip_kv_compact(self.c, b, pt, None if keep is None else ints(keep))
        self.o.compact(seqs, counts, paths, keep)
        self.check()

    def check(self):
        o = self.o
        assert self.c.page_table.tolist() == o.table
        assert self.c.seq_len.tolist() == o.len
        assert self.c.page_refs.tolist() == o.refs
        k, v = self.c.k.float().cpu().numpy(), self.c.v.float().cpu().numpy()
        for s in range(len(o.len)):                            # every committed row, in every layer and head
            for pos in range(o.len[s]):
                at = o.place(s, pos)
                for layer in range(self.layers):
                    name = o.rows[at] + 1000 * layer
                    assert (k[layer, at[0], :, at[1]] == name).all() and (v[layer, at[0], :, at[1]] == -name).all()

    def free(self, seqs):
        self.D.dip_kv_free(self.c, ints(seqs))
        self.o.free(seqs)
        self.check()

    def fork(self, src, dst):
        self.D.dip_kv_fork(self.c, ints(src), ints(dst))
        self.o.fork(src, dst)
        self.check()


@pytest.mark.parametrize("slot_major", [False, True])
@pytest.mark.parametrize("page", [1, 4, 16])
def test_pages_of_a_branching_decode(page, slot_major):
    c = Paged(n_pages=160 // page + 6, page=page, n_seqs=6, max_pages=48 // page + 1, slot_major=slot_major)
    c.check()
    c.step([2, 0], [13, 5])                                    # two prompts
    c.fork([2, 2, 0], [1, 3, 4])
    c.step([1, 3, 4], [4, 3, 2], [[0, 2], [0], [0, 1]], [2, 1, 2])
    c.step([2], [1])                                           # the source goes on: its last page is shared no more
    c.step([1, 2, 3], [7, 0, 6], [[0, 1, 4, 6], [], [0, 3, 5]], [4, 0, 3])
    c.free([1, 1, 99, -3])
    c.fork([3], [1])
    c.step([1, 3], [5, 5], [[0, 4], [0, 1, 2, 3, 4]], [2, 5])
    c.free([0, 2, 4])
    c.step([0, 5], [9, 1])
    c.free([0, 1, 2, 3, 4, 5])
    assert set(c.c.page_refs.tolist()) == {0}


def test_pages_run_out_and_tables_end():
    c = Paged(n_pages=7, page=4, n_seqs=5, max_pages=4, dtype=torch.bfloat16, layers=1)
    c.step([0, 1], [8, 5])                                     # 2 + 2 of 7
    c.step([2, 3, 4], [9, 4, 8])                               # 3 fit; what is behind does not
    c.step([0, 1], [9, 3])                                     # longer than the table; within its own page
    c.step([0, 1, 2], [1, 1, 3], [[0], [0], [0, 2]], [1, 1, 2])
    c.fork([0], [3])
    c.step([3], [4])                                           # nothing left


def test_reserve_many_entries_and_pages():
    c = Paged(n_pages=9000, page=1, n_seqs=1024, max_pages=40, hkv=1, layers=1)
    rng = np.random.default_rng(0)
    c.step(list(range(1024)), [int(x) for x in rng.integers(0, 9, 1024)])
    c.free([int(x) for x in rng.choice(1024, 400, replace=False)])
    live = [int(x) for x in rng.permutation(1024)[:700]]
    c.step(live, [int(x) for x in rng.integers(0, 7, 700)])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("slot_major", [False, True])
def test_copy_pages(dtype, slot_major):
    import paper_2412_01380_amd as D
    shape = (3, 9, 5, 16, 24)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(shape, generator=g, device="cuda").to(dtype) for _ in range(2))
    if slot_major:
        k, v = (t.transpose(2, 3).contiguous().transpose(2, 3) for t in (k, v))
    cache = D.KvCache(k, v, ints([[0]]), ints([0]), torch.zeros(9, dtype=torch.int32, device="cuda"))
    kk, vv = k.clone(), v.clone()
    D.dip_kv_copy_pages(cache, ints([1, 7, 2, -1, 3, 4]), ints([0, 8, 5, 6, 9, 4]))
    for a, b in [(1, 0), (7, 8), (2, 5)]:
        kk[:, b], vv[:, b] = kk[:, a].clone(), vv[:, a].clone()
    assert torch.equal(k, kk) and torch.equal(v, vv)


def test_compact_many_rows_and_strided_new_rows():
    # more rows than are in flight at once, most of them moved; rows taken out of a fused projection
    import paper_2412_01380_amd as D
    rng = np.random.default_rng(2)
    k, v = (torch.zeros(2, 12, 3, 16, 64, device="cuda") for _ in range(2))
    cache = D.KvCache(k, v, ints([[-1] * 10, [-1] * 10]), ints([0, 0]), torch.zeros(12, dtype=torch.int32, device="cuda"))
    rows = [90, 70]
    b = D.Batch(starts(rows), 160, 90, seqs=ints([1, 0]))
    ws = workspace(D.dip_kv_reserve_workspace_bytes(cache, b))
    D.dip_kv_reserve(cache, b, None, ws)
    fused = torch.randn(2, 160, 3 * 3 * 64, device="cuda")
    k_new, v_new = (fused[:, :, i * 192:(i + 1) * 192].unflatten(2, (3, 64)) for i in (1, 2))
    D.dip_kv_append(cache, 0, b, k_new, v_new)
    paths = [sorted(rng.choice(r, size=m, replace=False).tolist()) for r, m in zip(rows, (61, 70))]
    flat = [x for p, r in zip(paths, rows) for x in p + [-1] * (r - len(p))]
    D.dip_kv_compact(cache, b, ints(flat), ints([61, 70]))
    assert cache.seq_len.tolist() == [70, 61]
    for e, (seq, first) in enumerate([(1, 0), (0, 90)]):
        table = cache.page_table[seq].tolist()
        for j, src in enumerate(paths[e]):
            pg, sl = table[j // 16], j % 16
            assert torch.equal(k[:, pg, :, sl], k_new[:, first + src]) and torch.equal(v[:, pg, :, sl], v_new[:, first + src])


# ---- shares, large batches, long tables --------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_batches_of_more_entries_than_a_wavefront_has_lanes(dtype):
    rng = np.random.default_rng(6)
    lens = [int(x) for x in rng.integers(0, 300, 150)]
    lens[70], lens[149] = 2600, 1500
    rows = [int(x) for x in rng.integers(0, 4, 150)]
    rows[0], rows[70], rows[149] = 0, 2, 3
    s = Setup(dtype, lens, rows, 2, 1, 64, 16, seed=4)
    for window, sinks in [(0, 0), (200, 5)]:
        s.check(s.run(window, sinks), window, sinks)
    par = [random_tree(rng, n) for n in rows]
    s.check(s.run(0, 0, par), 0, 0, par)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(128, 16), (96, 64), (64, 1)])
def test_wide_trees_in_shares(dtype, d, page):
    rng = np.random.default_rng(d)
    s = Setup(dtype, [3000, 700], [64, 50], 8, 2, d, page, seed=d)
    par = [random_tree(rng, 64, absent=True), random_tree(rng, 50)]
    for window, sinks in [(0, 0), (1500, 70)]:
        s.check(s.run(window, sinks, par), window, sinks, par)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 96, 128])
def test_pieces_of_prompts(dtype, d):
    s = Setup(dtype, [1500, 0, 64], [200, 150, 129], 4, 2, d, 32, slot_major=True, seed=d)
    for window, sinks in [(0, 0), (500, 70), (600, 1), (64, 0), (3, 100)]:
        s.check(s.run(window, sinks), window, sinks)


@pytest.mark.parametrize("page", [1, 8])
def test_one_token_over_many_small_pages(page):
    s = Setup("bf16", [9000, 4097], [1, 2], 4, 1, 128, page, seed=3)
    s.check(s.run())


def test_prompts_where_something_is_not_finite():
    clean = Setup("bf16", [900], [130], 8, 2, 128, 16, seed=8)
    ref = clean.run(700, 4)
    s = Setup("bf16", [900], [130], 8, 2, 128, 16, seed=8)
    for pos in (10, 150, 200):                       # in front of every row's window
        s.put(0, pos, NAN)
    assert torch.equal(s.run(700, 4), ref)
    s.put(0, 960, math.inf)                          # row 60: seen by the rows from there on
    out = s.run(700, 4)
    assert torch.equal(out[:60], ref[:60])
    assert not torch.isfinite(out[60:].float()).all(-1).any()
    s.put(0, 960, float(s.k[0][959, 0, 0]))
    s.put(0, 600, NAN, "v")                          # seen by all of them: in whole tiles it goes where it belongs
    out = s.run(700, 4)
    assert torch.isnan(out.float()).all()


def test_shares_of_wide_trees_in_a_graph():
    s = Setup("bf16", [2500, 40], [40, 33], 8, 2, 128, 16, seed=2)
    rng = np.random.default_rng(0)
    par = [random_tree(rng, n) for n in s.rows]
    q, out, ws = s.q.cuda(), torch.empty(73, 8, 128, dtype=torch.bfloat16, device="cuda"), workspace(64 << 20)
    parents = ints([x for p in par for x in p])
    import paper_2412_01380_amd as D
    call = lambda o: D.dip_tree_attention(s.cache, 1, s.batch, parents, q, 0.1, 0, 0, o, ws)
    call(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for n in (2500, 100, 1800, 0):
        s.cache.seq_len[s.seqs[0]] = n
        eager = torch.empty_like(out)
        call(eager)
        out.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


def test_verify_in_a_graph_and_many_entries():
    import paper_2412_01380_amd as D
    rng = np.random.default_rng(5)
    trees = [random_tree(rng, int(n)) for n in rng.integers(1, 9, 90)]
    p, q, tokens, u, us = verify_inputs(rng, trees, 5000)
    check_verify(trees, p, q, tokens, u, us, 3)
    rows = [len(t) for t in trees]
    b = D.Batch(starts(rows), sum(rows), max(rows))
    keep, path, token = (torch.zeros(m, dtype=torch.int32, device="cuda") for m in (90, sum(rows), 90))
    ws = workspace(D.dip_verify_tree_workspace_bytes(b, 5000, 3))
    args = (ints(tokens), ints([x for t in trees for x in t]), p.cuda(), q.cuda(), torch.from_numpy(u).cuda(),
            torch.from_numpy(us).cuda())
    call = lambda: D.dip_verify_tree(b, *args, 3, keep, path, token, ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        args[4].copy_(torch.from_numpy(rng.random(sum(rows)).astype(np.float32)))
        call()
        eager = [t.clone() for t in (keep, path, token)]
        for t in (keep, path, token):
            t.fill_(-5)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, (keep, path, token)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("rows", [[1, 1], [8, 5], [33, 64]])
def test_contexts_that_may_be_long(dtype, d, rows):
    """Tables for far more keys than there are, and no bound on the lengths: the loads and the cut for large calls."""
    import paper_2412_01380_amd as D
    s = Setup(dtype, [1200, 77], rows, 8, 2, d, 16, seed=d + rows[0])
    table = torch.full((len(s.table), 8192), -1, dtype=torch.int32)
    table[:, :s.max_pages] = s.table
    s.cache = D.KvCache(s.cache.k, s.cache.v, table.cuda(), s.cache.seq_len, s.cache.page_refs)
    s.batch = D.Batch(starts(rows), sum(rows), max(rows), seqs=ints(s.seqs))
    par = [random_tree(np.random.default_rng(d), n) for n in rows]
    for window, sinks in [(0, 0), (100000, 3)]:
        s.check(s.run(window, sinks), window, sinks)
        s.check(s.run(window, sinks, par), window, sinks, par)
