"""What a bf16 cache costs in precision: the output's own rounding and hardly anything else, whichever kernel runs."""
import math

import numpy as np
import pytest

from oracle import decode_oracle as O
from test_gpu_decode import Setup, random_tree

pytestmark = pytest.mark.gpu


def check_rounding(s, out, window, sinks, parents=None):
    """An output is rounded to bf16 once, by up to 2^-8 of itself.  The weights' two terms hold 15 bits and more of them
    (2^-14 of sum p |v| bounds their rounding and that of their sum); scores, exponentials and sums are fp32 as in
    Setup.check."""
    got, at = out.double().cpu().numpy(), 0
    for i, (n, r) in enumerate(zip(s.lens, s.rows)):
        sees = O.visible(n, r, window, sinks, None if parents is None else parents[i])
        ref, mag, big = O.attend(s.q64[at:at + r], s.k[i], s.v[i], sees, 1 / math.sqrt(s.d))
        dz = (big * (s.d / 4 + 8) + 64)[..., None] * 2.0 ** -24
        inner = mag * (2 * dz + (4 * math.sqrt(n + r) + 32) * 2.0 ** -24 + 2.0 ** -14) + 1e-30
        err = np.abs(got[at:at + r] - ref)
        bound = inner + (np.abs(ref) + inner) * 2.0 ** -8
        assert (err <= bound).all(), (i, float((err / bound).max()), float((err > bound).mean()))
        at += r


# few keys carry a row (keys three times as long) or all of them alike; one block of rows and several, edges and middles
@pytest.mark.parametrize("wide", [1.0, 3.0])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("lens,rows", [([900, 40], [130, 70]), ([3000, 300], [5, 8]), ([2100, 700], [64, 40]), ([0], [200])])
def test_weights_lose_nothing_that_shows(lens, rows, d, wide):
    s = Setup("bf16", lens, rows, 8, 2, d, 16, seed=d, wide=wide)
    for window, sinks in [(0, 0), (600, 4), (64, 0)]:
        check_rounding(s, s.run(window, sinks), window, sinks)
    if max(rows) <= 64:
        par = [random_tree(np.random.default_rng(d), n) for n in rows]
        check_rounding(s, s.run(0, 0, par), 0, 0, par)


def test_a_token_is_as_exact_beside_a_prompt_as_alone():
    s = Setup("bf16", [1500, 260, 9], [1, 180, 1], 8, 2, 128, 16, seed=2, wide=3.0)
    for window, sinks in [(0, 0), (300, 4)]:
        check_rounding(s, s.run(window, sinks), window, sinks)
