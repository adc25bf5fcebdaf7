"""Draws of a row of which whole chunks lie so far below its maximum that they weigh nothing."""
import math

import pytest
import torch

from test_gpu_decode import DT, ints
from test_gpu_sample import check, floats, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("u", [0.0, 2.0 ** -149, 0.5, 1 - 2.0 ** -24])
@pytest.mark.parametrize("below", [63.5, 63.75, 64.0, 70.0, 1e30])
def test_a_chunk_that_weighs_nothing(below, u, dtype):
    # a row of -1 only where there is no word above -inf; top_k as many as there are words: the same by another way
    for first, last in ((0.0, -below), (-below, 0.0), (1.0, 1.0 - below)):
        x = torch.full((2, 20000), -math.inf)
        x[:, :8192], x[:, 8192], x[:, 8193:12288], x[:, 19999] = last, first, last, max(first, last)
        x = x.to(DT[dtype]).cuda()
        us = floats([u, u])
        for how in (None, dict(top_k=ints([20000, 20000 - 1])), dict(top_p=floats([1.0, 1 - 2.0 ** -24]))):
            token, probs = run(x, us, torch.float32, how)
            assert (token >= 0).all()
            check(x, us, token, probs, how)
