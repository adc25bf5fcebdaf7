"""Attention where max_len, or the end of the page table, lies below a sequence's rows: what lies from there on is seen
by nobody, wherever in a tile that is."""
import math

import numpy as np
import pytest

from oracle import decode_oracle as O
from test_gpu_decode import Setup, ints, random_tree, starts

pytestmark = pytest.mark.gpu


def check_cut(s, out, cut, window, sinks, parents=None):
    """Setup.check with nothing seen from position `cut` on."""
    got, at = out.double().cpu().numpy(), 0
    for i, (n, r) in enumerate(zip(s.lens, s.rows)):
        sees = O.visible(n, r, window, sinks, None if parents is None else parents[i])
        sees[:, cut:] = False
        ref, mag, big = O.attend(s.q64[at:at + r], s.k[i], s.v[i], sees, 1 / math.sqrt(s.d))
        dz = (big * (s.d / 4 + 8) + 64)[..., None] * 2.0 ** -24
        bound = mag * (2 * dz + (4 * math.sqrt(n + r) + 32) * 2.0 ** -24) + 1e-30
        if s.dtype == "bf16":
            bound = bound + (mag + np.abs(ref)) * 2.0 ** -8.9
        err = np.abs(got[at:at + r] - ref)
        assert (err <= bound).all(), (cut, i, window, float((err / bound).max()))
        assert not got[at:at + r][~sees.any(1)].any()
        at += r


CASES = [
    # lens, rows, hq, hkv, d, page
    ([38, 3], [4, 2], 4, 2, 128, 16),
    ([61, 200], [30, 9], 8, 2, 64, 8),
    ([150, 90], [64, 50], 8, 2, 128, 32),
    ([77, 130], [64, 33], 6, 3, 96, 64),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_nothing_is_seen_from_max_len_on(case, dtype):
    import paper_2412_01380_amd as D
    lens, rows, hq, hkv, d, page = case
    s = Setup(dtype, lens, rows, hq, hkv, d, page, seed=3)
    rng = np.random.default_rng(1)
    par = [random_tree(rng, n, absent=True) for n in rows]
    most = max(n + r for n, r in zip(lens, rows))
    # inside the rows, at their start, inside what was committed, behind all but a few positions
    for cut in sorted({most - 1, lens[0] + 2, lens[0], lens[0] - 5, lens[1] + 1, 33, 1}):
        b = D.Batch(starts(rows), sum(rows), max(rows), seqs=ints(s.seqs), max_len=cut)
        for window, sinks in [(0, 0), (20, 3), (6, 0)]:
            check_cut(s, s.run(window, sinks, batch=b), cut, window, sinks)
            check_cut(s, s.run(window, sinks, par, batch=b), cut, window, sinks, par)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [[9, 1], [70, 20]])
def test_rows_behind_the_end_of_the_table(dtype, rows):
    # tables of 23 positions, no multiple of a tile: rows from there on have no place in them
    import paper_2412_01380_amd as D
    s = Setup(dtype, [20, 2], rows, 4, 2, 64, 1, seed=5)
    table = s.cache.page_table[:, :23].contiguous()
    s.cache = D.KvCache(s.cache.k, s.cache.v, table, s.cache.seq_len, s.cache.page_refs)
    s.batch = D.Batch(starts(rows), sum(rows), max(rows), seqs=ints(s.seqs))
    par = [random_tree(np.random.default_rng(0), min(n, 64)) for n in rows]
    for window, sinks in [(0, 0), (9, 2)]:
        check_cut(s, s.run(window, sinks), 23, window, sinks)
        if max(rows) <= 64:
            check_cut(s, s.run(window, sinks, par), 23, window, sinks, par)
