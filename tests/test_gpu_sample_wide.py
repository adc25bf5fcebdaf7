"""Cuts by top_k and top_p together where they lie far below the maximum, among words that weigh next to nothing each but
something together; and draws where a whole chunk of a row weighs nothing."""
import math

import numpy as np
import pytest
import torch

from test_gpu_decode import DT, ints
from test_gpu_sample import CLOSE, floats, run

pytestmark = pytest.mark.gpu

# Weights are accurate to 2^-26, and so are sums of them: what one sum is compared with, a part of another, may be 2^-25 off.
PART = 2.0 ** -25


def check_ranges(x, u, token, probs, how):
    """The kept words are the first n in order of (logit, number), n within what the accuracy of sums leaves open; the token is one at
    which the running sum passes u, and a probability within its roundings (as in test_gpu_sample.check)."""
    for i, row in enumerate(x.double().cpu().numpy()):
        row = row + 0.0
        k, part = int(how["top_k"][i]), float(how["top_p"][i])
        least = float(how["min_p"][i]) if "min_p" in how else 0.0
        order = np.argsort(-row, kind="stable")
        order = order[row[order] > -np.inf][:k if k > 0 else None]
        w = np.exp(row[order] - row[order[0]])
        sums = np.cumsum(w)
        most = [int(np.searchsorted(sums, part * y * sums[-1])) + 1 if part < 1 else len(w) for y in (1 - PART, 1 + PART)]
        if least > 0:
            most = [max(1, min(n, int((w >= least * y).sum()))) for n, y in zip(most, (1 + PART, 1 - PART))]
        got = probs[i].double().cpu().numpy()
        n = int((got > 0).sum())
        assert most[0] <= n <= most[1], (i, n, most)
        assert (got[order[:n]] > 0).all(), i
        kept = np.zeros(len(row))
        kept[order[:n]] = w[:n]
        run_sum = np.cumsum(kept) / kept.sum()
        lo = int(np.searchsorted(run_sum, float(u[i]) - CLOSE, side="right"))
        hi = min(int(np.searchsorted(run_sum, float(u[i]) + CLOSE, side="right")), int(np.nonzero(kept)[0][-1]))
        assert lo <= int(token[i]) <= hi and kept[int(token[i])] > 0, (i, int(token[i]), lo, hi)
        p = kept / kept.sum()
        assert (np.abs(got - p) <= p * 5 * 2.0 ** -24 + 2.0 ** -126).all(), (i, float(np.abs(got / np.maximum(p, 1e-300) - 1)[p > 0].max()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v,low,part", [(128256, -20.3, 0.9999), (128256, -20.3, 0.99995), (128256, -14.0, 0.97), (40000, -30.0, 1 - 2.0 ** -24),
                                        (1 << 20, -22.0, 0.99985), (1 << 24, -26.25, 0.99995)])
def test_one_word_above_many_equal_ones(v, low, part, dtype):
    x = torch.full((3, v), low, device="cuda")
    x[0, 7], x[1, v // 2], x[2, v - 1] = 0.0, 0.0, 0.0
    if v == 1 << 24:
        x = x[1:2]
    n = len(x)
    x, u = x.to(DT[dtype]), floats([1 - 2.0 ** -14, 0.0, 0.9999999][:n])
    how = dict(top_k=ints([v - 1, v - 5, v // 2 + 9][:n]), top_p=floats([part] * n))
    token, probs = run(x, u, torch.float32, how)
    check_ranges(x, u, token, probs, how)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", [3000, 70001, 300007])
def test_both_rules_over_many_bins(v, dtype):
    # a few words near the maximum, the others spread over 30 nats: of top_k's cut and top_p's any bin, list or row
    g = torch.Generator().manual_seed(v)
    n = 12
    x = -2.0 - 28.0 * torch.rand(n, v, generator=g) ** torch.linspace(0.1, 1.5, n)[:, None]
    x[:, 5] = 0.0
    x[3] = x[3].round()
    x[torch.rand(n, v, generator=g) < 0.05] = -math.inf
    x[7] -= 40.0
    x[8, :5] = -70.0
    x = x.to(DT[dtype]).cuda()
    u = torch.rand(n, generator=g).cuda()
    how = dict(top_k=(v * (0.1 + 0.9 * torch.rand(n, generator=g))).int().cuda(),
               top_p=(1 - 0.1 * torch.rand(n, generator=g) ** 6).clamp(max=1 - 2.0 ** -24).cuda())
    token, probs = run(x, u, torch.float32, how)
    check_ranges(x, u, token, probs, how)
    how["min_p"] = torch.exp(-30 * torch.rand(n, generator=g)).cuda()
    token, probs = run(x, u, torch.float32, how)
    check_ranges(x, u, token, probs, how)
