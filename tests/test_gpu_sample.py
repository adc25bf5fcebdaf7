"""Tokens and probabilities from logits against the 64-bit oracle: every rule alone and together, ties, rows of any odd
length and stride, infinities, temperatures from next to nothing to infinite, rows whose cut lies far down."""
import math

import numpy as np
import pytest
import torch

from oracle import decode_oracle as O
from test_gpu_decode import DT, NAN, ints, workspace

pytestmark = pytest.mark.gpu

# weights are held to 2^-27 and the running sums of them are exact: a draw or a cut nearer than this to a border may go
# either way
CLOSE = 2.0 ** -26


def floats(v):
    return torch.tensor(v, dtype=torch.float32, device="cuda")


def run(x, u=None, probs=torch.float32, how=None, ws=None, stream=None, out=None):
    import paper_2412_01380_amd as D
    n, v = x.shape
    ws = workspace(D.dip_sample_workspace_bytes(n, v)) if ws is None else ws
    token = torch.full((n,), -7, dtype=torch.int32, device="cuda") if u is not None else None
    if out is None and probs is not None:
        out = torch.full((n, v), NAN, dtype=probs, device="cuda")
    D.dip_sample(x, u, token, out, ws, stream=stream, **(how or {}))
    return token, out


def check(x, u, token, probs, how=None):
    """Tokens equal, the same words kept, and each probability within its roundings: the exponential and its argument (2), the
    sum's reciprocal, a product (2), and the weights' own 2^-27 in the sum: 5 of 2^-24; then that of its type."""
    rows = x.double().cpu().numpy()
    h = {k: v.double().cpu().numpy() for k, v in (how or {}).items() if v is not None}
    got = probs.double().cpu().numpy() if probs is not None else None
    for i, row in enumerate(rows):
        T, k = h["temperature"][i] if "temperature" in h else 1.0, int(h["top_k"][i]) if "top_k" in h else 0
        part, least = h["top_p"][i] if "top_p" in h else 1.0, h["min_p"][i] if "min_p" in h else 0.0
        w, close = O.sample(row, T, k, part, least)
        if w is None:
            assert token is None or token[i] == -1
            assert got is None or not got[i].any()
            continue
        if close <= CLOSE and got is not None:            # a cut next to a border: on either side of it
            near = [1.0, 1 - 2 * CLOSE, 1 + 2 * CLOSE]
            for a, b in [(a, b) for a in near for b in near]:
                v, _ = O.sample(row, T, k, part * a if part < 1 else part, min(least, 1.0) * b if least > 0 else least)
                if (v > 0).sum() == (got[i] > 0).sum():
                    w = v
                    break
        sums = np.cumsum(w) / w.sum()
        if token is not None:
            may = [int(np.nonzero(sums > y)[0][0]) if (sums > y).any() else int(np.nonzero(w)[0][-1])
                   for y in (float(u[i]) - CLOSE, float(u[i]), float(u[i]) + CLOSE)]
            assert int(token[i]) in may and w[int(token[i])] > 0, (i, int(token[i]), may)
        if got is not None:
            p = w / w.sum()
            half = 2.0 ** -8 if probs.dtype == torch.bfloat16 else 0.0
            tiny = 2.0 ** -126
            assert ((got[i] > 0) == (p > 0))[(p >= tiny) | (w == 0)].all(), i
            assert (np.abs(got[i] - p) <= p * (5 * 2.0 ** -24 + half) + tiny).all(), (i, np.abs(got[i] / np.maximum(p, 1e-300) - 1).max())


def logits(n, v, dtype, seed, sigma=2.5, banned=0.02):
    g = torch.Generator().manual_seed(seed)
    x = sigma * torch.randn(n, v, generator=g)
    x[torch.rand(n, v, generator=g) < banned] = -math.inf
    return x.to(DT[dtype]).cuda(), torch.rand(n, generator=g).cuda()


HOWS = {
    "none": {}, "warm": dict(temperature=[0.7, 1.3, 0.01, 5.0, 1.0]), "greedy": dict(temperature=[0.0, -1.0, NAN, 1.0, 0.5]),
    "k": dict(top_k=[1, 2, 50, 700, 0]), "p": dict(top_p=[0.1, 0.5, 0.9, 0.999, 1.0]), "min": dict(min_p=[0.5, 0.05, 0.001, 1.0, 0.0]),
    "kp": dict(top_k=[3, 40, 200, 1000, -5], top_p=[0.9, 0.8, 0.99, 0.3, 0.95]),
    "all": dict(temperature=[0.8, 1.1, 0.0, 1.5, 0.6], top_k=[40, 0, 10, 500, 20], top_p=[0.95, 0.9, 0.5, 0.8, 1.0],
                min_p=[0.02, 0.1, 0.5, 0.0, 0.05]),
    "odd": dict(top_k=[2147483647, -2147483648, 5, 5, 5], top_p=[NAN, 2.0, -1.0, 0.0, math.inf], min_p=[NAN, -1.0, 0.0, 7.0, 1.0]),
    "tiny": dict(temperature=[1e-3, 1e-7, 1e-30, 1e-44, math.inf], top_k=[5, 60, 3, 2, 17]),
    "hot": dict(temperature=[100.0, math.inf, 1e30, 3.0, 1.0], top_p=[0.9, 0.4712389, 0.2345678, 0.999, 0.9], min_p=[0.0, 0.5, 0.0, 0.001, 0.0]),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", [1, 2, 17, 1000, 8191, 8192, 8193, 32064, 70001])
@pytest.mark.parametrize("name", list(HOWS))
def test_rules(name, v, dtype):
    x, u = logits(5, v, dtype, seed=v, banned=0.02 if v > 2 else 0.0)
    how = {k: (ints if k == "top_k" else floats)(a) for k, a in HOWS[name].items()}
    token, probs = run(x, u, torch.float32, how)
    check(x, u, token, probs, how)
    alone, _ = run(x, u, None, how)
    assert torch.equal(alone, token)
    _, short = run(x, None, torch.bfloat16, how)
    assert torch.equal(short, probs.bfloat16())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", [9000, 100003])
def test_ties_go_to_the_lowest_numbers(v, dtype):
    # a few values only: every cut falls among thousands of equal logits, more than a row's list holds
    g = torch.Generator().manual_seed(3)
    x = torch.randint(-2, 2, (6, v), generator=g).to(DT[dtype]).cuda()
    x[5] = -0.0
    x[5, ::3] = 0.0
    how = dict(top_k=ints([3, 2500, v // 2, 0, 0, 1000]), top_p=floats([1.0, 0.73, 0.9, 0.61, 0.37, 1.0]), min_p=floats([0, 0, 0, 0, 0.2, 0]))
    u = floats([0.1, 0.99, 0.5, 0.7, 0.3, 0.9995])
    token, probs = run(x, u, torch.float32, how)
    check(x, u, token, probs, how)
    assert torch.nonzero(probs[5])[:, 0].tolist() == list(range(1000))
    # exact halves: 5 of 10 equal words come to one half
    x = torch.zeros(1, 10, dtype=DT[dtype], device="cuda")
    _, probs = run(x, None, torch.float32, dict(top_p=floats([0.5])))
    assert probs[0].tolist() == [0.20000000298023224] * 5 + [0.0] * 5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cuts_far_down(dtype):
    # one word far above all others: top_k's cut lies hundreds of nats below it; and at the lowest finite numbers
    x, u = logits(4, 20000, dtype, 5)
    x[0, 777] = 1000.0
    x[1] *= 200
    x[2, 5], x[2, 6] = torch.finfo(DT[dtype]).max, torch.finfo(DT[dtype]).min
    x[3] = torch.finfo(DT[dtype]).min
    x[3, 9999] = 3.0
    how = dict(top_k=ints([30, 5000, 19000, 7]), top_p=floats([1.0, 1.0, 0.99, 1.0]))
    token, probs = run(x, u, torch.float32, how)
    check(x, u, token, probs, how)
    import paper_2412_01380_amd as D
    assert int(token[0]) == 777 and int(token[3]) == 9999 and D.DIP_OK == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_not_finite(dtype):
    x, u = logits(8, 12345, dtype, 6)
    x[0] = -math.inf
    x[1] = NAN
    x[2, 4000:] = NAN
    x[3, 7] = math.inf
    x[4, 7], x[4, 9000], x[4, 12000] = math.inf, math.inf, NAN
    x[5] = -math.inf
    x[5, 12344] = -3.0
    x[6] = math.inf
    for how in ({}, dict(top_k=ints([5] * 8), top_p=floats([0.9] * 8)), dict(min_p=floats([0.1] * 8)), dict(temperature=floats([0.0] * 8)),
                dict(temperature=floats([math.inf] * 8), top_k=ints([3] * 8))):
        token, probs = run(x, u, torch.float32, how)
        check(x, u, token, probs, how)
    token, probs = run(x, None, torch.float32)
    assert probs[4, 7] == 0.5 and probs[4, 9000] == 0.5 and probs[3, 7] == 1.0


def test_views_one_row_and_in_place():
    x, u = logits(5, 3001, "f32", 8)
    wide = torch.full((5, 9005), NAN, device="cuda")
    wide[:, 1:3002] = x                                        # rows that start anywhere, and a column of the same array out
    out = wide[:, 4003:7004]
    how = dict(top_p=floats([0.8] * 5))
    token, probs = run(wide[:, 1:3002], u, None, how, out=out)
    check(x, u, token, probs, how)
    assert wide[:, 0].isnan().all() and wide[:, 3002:4003].isnan().all() and wide[:, 7004:].isnan().all()
    for dt in ("bf16", "f32"):
        x, u = logits(5, 3001, dt, 9)
        token, probs = run(x, u, x.dtype, how)
        again = x.clone()
        token2, probs2 = run(again, u, None, how, out=again)
        assert torch.equal(token, token2) and torch.equal(probs, again)
    one, u1 = logits(1, 128256, "bf16", 10)
    how = dict(top_k=ints([40]), top_p=floats([0.9]))
    token, probs = run(one, u1, torch.float32, how)
    check(one, u1, token, probs, how)


def test_a_vocabulary_of_millions():
    x, u = logits(2, 5000011, "bf16", 11)
    for how in ({}, dict(top_k=ints([100, 3000000]), top_p=floats([0.9, 0.99]))):
        token, probs = run(x, u, torch.float32, how)
        check(x, u, token, probs, how)


def test_the_same_bits_every_time_and_in_a_graph():
    x, u = logits(40, 50001, "bf16", 12)
    how = dict(temperature=floats([0.5 + 0.05 * i for i in range(40)]), top_k=ints([7 * i for i in range(40)]),
               top_p=floats([1 - 0.02 * i for i in range(40)]), min_p=floats([0.01 * (i % 5) for i in range(40)]))
    import paper_2412_01380_amd as D
    ws = workspace(D.dip_sample_workspace_bytes(40, 50001))
    token, probs = run(x, u, torch.float32, how, ws)
    t2, p2 = torch.empty_like(token), torch.empty_like(probs)
    t3, p3 = torch.empty_like(token), torch.empty_like(probs)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]        # two graphs that share a workspace
    for graph, t, p in zip(graphs, (t2, t3), (p2, p3)):
        with torch.cuda.graph(graph):
            D.dip_sample(x, u, t, p, ws, **how)
    for i in range(4):
        keep = x.clone()
        if i:
            x.copy_(x.roll(1, 0))
        token, probs = run(x, u, torch.float32, how, ws)
        for graph, t, p in zip(graphs, (t2, t3), (p2, p3)):
            t.fill_(-7), p.fill_(NAN)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(t, token) and torch.equal(p, probs)
        del keep


def test_draws_follow_the_probabilities():
    # all numbers of a fine grid: word x is drawn for just its share of them
    x, _ = logits(1, 300, "f32", 13, banned=0.1)
    n = 20000
    u = (torch.arange(n, device="cuda") + 0.5) / n
    token, probs = run(x.expand(n, 300).contiguous(), u, torch.float32, dict(top_p=floats([0.95] * n)))
    counts = torch.bincount(token.long(), minlength=300).double() / n
    assert (counts - probs[0].double()).abs().max() <= 1.0 / n + 1e-6


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows_of_any_settings(dtype):
    g = torch.Generator().manual_seed(14)
    n, v = 1500, 257
    x = torch.randn(n, v, generator=g) * torch.exp(3 * torch.rand(n, 1, generator=g))
    x[::3] = (2 * x[::3]).round() / 2                          # a third of the rows full of ties
    x[torch.rand(n, v, generator=g) < 0.3 * torch.rand(n, 1, generator=g)] = -math.inf
    x[7::50, 3] = math.inf
    x = x.to(DT[dtype]).cuda()
    some = lambda lo, hi: lo + (hi - lo) * torch.rand(n, generator=g)
    how = dict(temperature=some(-0.1, 2.0), top_k=(some(0, 1) ** 2 * 300).int() - 20, top_p=some(0.0, 1.2), min_p=some(-0.1, 0.3) ** 3)
    how = {k: t.cuda() for k, t in how.items()}
    u = torch.rand(n, generator=g).cuda()
    token, probs = run(x, u, torch.float32, how)
    check(x, u, token, probs, how)
    for left in ("top_k", "top_p", "min_p"):
        part = {k: t for k, t in how.items() if k != left}
        token, probs = run(x, u, torch.float32, part)
        check(x, u, token, probs, part)


def test_rows_as_many_as_there_may_be():
    x, u = logits(65535, 40, "bf16", 15)
    token, probs = run(x, u, torch.bfloat16, dict(top_k=ints([3] * 65535)))
    some = list(range(0, 65535, 997)) + [65534]
    check(x[some], u[some], token[some], probs[some], dict(top_k=ints([3] * len(some))))
