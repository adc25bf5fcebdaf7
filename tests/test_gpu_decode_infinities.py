"""Values that are not finite: a channel that a row sees one of is what the sum gives -- infinite, or NaN where there is
one, or infinities of both signs --, all other channels are as they were, wherever in a tile the key lies."""
import math

import numpy as np
import pytest
import torch

from oracle import decode_oracle as O
from test_gpu_decode import Setup, random_tree

pytestmark = pytest.mark.gpu


def check_channels(s, out, window, sinks, parents=None):
    got, at = out.double().cpu().numpy(), 0
    for i, (n, r) in enumerate(zip(s.lens, s.rows)):
        sees = O.visible(n, r, window, sinks, None if parents is None else parents[i])
        with np.errstate(invalid="ignore"):
            ref, mag, big = O.attend(s.q64[at:at + r], s.k[i], s.v[i], sees, 1 / math.sqrt(s.d))
        dz = (big * (s.d / 4 + 8) + 64)[..., None] * 2.0 ** -24
        fine, x = np.isfinite(ref), got[at:at + r]
        mag = np.where(fine, mag, 0.0)
        bound = mag * (2 * dz + (4 * math.sqrt(n + r) + 32) * 2.0 ** -24) + 1e-30
        if s.dtype == "bf16":
            bound = bound + (mag + np.abs(np.where(fine, ref, 0.0))) * 2.0 ** -8.9
        nans, signs = bool((np.isnan(x) == np.isnan(ref)).all()), bool((x[np.isinf(ref)] == ref[np.isinf(ref)]).all())
        near = bool((np.abs(x[fine] - ref[fine]) <= bound[fine]).all())
        assert (nans, signs, near) == (True, True, True), (i, window)
        at += r


def spoil(s, entry, pos, channel, value):
    """One channel of the value at one position, all heads."""
    page = s.cache.k.shape[3]
    pg, sl = int(s.table[s.seqs[entry], pos // page]), pos % page
    s.cache.v[s.layer, pg, :, sl, channel] = value
    s.v[entry][pos][:, channel] = value


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(64, 16), (96, 8), (128, 64)])
@pytest.mark.parametrize("lens,rows", [([700, 90], [3, 5]), ([700, 90], [64, 30]), ([700, 90], [150, 70])])
def test_infinite_channels(lens, rows, d, page, dtype):
    s = Setup(dtype, lens, rows, 8, 2, d, page, seed=d)
    inf, nan = math.inf, math.nan
    # in the middle of the past, at a window's edge, in the sinks, among the rows themselves
    for pos, channel, value in [(300, 5, inf), (301, 6, -inf), (320, 7, inf), (331, 7, -inf), (340, 17, nan), (1, 33, inf),
                                (lens[0] - 30, d - 1, -inf), (lens[0] + 1, 0, inf), (lens[0] + 2, 1, nan), (lens[0] + 2, 2, -inf),
                                (lens[0] + rows[0] - 1, 40, inf)]:
        spoil(s, 0, pos, channel, value)
    for pos, channel, value in [(0, 3, inf), (64, 4, -inf), (91, 5, nan), (92, 5, inf)]:
        spoil(s, 1, pos, channel, value)
    for window, sinks in [(0, 0), (400, 4), (31, 0), (405, 2)]:
        check_channels(s, s.run(window, sinks), window, sinks)
    if max(rows) <= 64:
        par = [random_tree(np.random.default_rng(d), n, absent=True) for n in rows]
        for window, sinks in [(0, 0), (400, 4)]:
            check_channels(s, s.run(window, sinks, par), window, sinks, par)


def test_shares_with_infinite_channels():
    for dtype in ("bf16", "f32"):
        for rows in ([2, 1], [64, 40]):
            s = Setup(dtype, [4000, 77], rows, 8, 2, 128, 16, seed=1)
            for pos, channel, value in [(3, 9, math.inf), (2000, 10, -math.inf), (3999, 11, math.inf), (100, 11, -math.inf), (3100, 12, math.nan)]:
                spoil(s, 0, pos, channel, value)
            check_channels(s, s.run(0, 0), 0, 0)
            check_channels(s, s.run(1500, 4), 1500, 4)
