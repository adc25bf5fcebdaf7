"""Host-side checks of dip_sample: bad arguments are refused before the HIP runtime is touched, workspaces have sizes, and
the oracle agrees with rows worked by hand."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import decode_oracle as O

FAKE = 0x10000


@pytest.fixture(scope="module")
def D():
    import paper_2412_01380_amd as D
    return D


def test_arguments_are_refused(D):
    def call(logits=FAKE, stride=100, dtype=0, rows=3, vocab=100, u=FAKE, token=FAKE, probs=None, ps=100, pd=0, ws=FAKE, n=1 << 40):
        return D.lib.dip_sample(logits, stride, dtype, rows, vocab, None, u, token, probs, ps, pd, ws, n, None)

    I, U, W = D.DIP_ERR_INVALID_ARG, D.DIP_ERR_UNSUPPORTED, D.DIP_ERR_WORKSPACE
    assert call(logits=None) == I
    assert call(token=None) == I and call(u=None) == I
    assert call(rows=0) == I and call(vocab=0) == I
    assert call(rows=65536) == U and call(vocab=(1 << 24) + 1, stride=1 << 25) == U
    assert call(dtype=2) == U and call(probs=0x90000, pd=2) == U
    assert call(stride=99) == I and call(probs=0x90000, ps=99) == I
    assert call(logits=FAKE + 2) == U and call(probs=0x90002) == U
    assert call(probs=FAKE + 4) == I and call(probs=FAKE, pd=1) == I and call(probs=FAKE, ps=101) == I
    assert call(probs=FAKE + 1200 - 4) == I
    need = D.dip_sample_workspace_bytes(3, 100)
    assert call(ws=None) == W and call(ws=FAKE + 16) == W and call(n=need - 1) == W
    assert D.dip_sample_workspace_bytes(0, 100) == 0 and D.dip_sample_workspace_bytes(1, 1 << 25) == 0
    assert D.dip_sample_workspace_bytes(1, 1 << 24) > 0
    assert call(probs=0x90000, token=None, u=None, n=8) == W             # (probabilities alone are a call)


def test_oracle_by_hand():
    x = np.log(np.array([0.1, 0.4, 0.1, 0.3, 0.1]))
    w = lambda *a, **k: np.nonzero(O.sample(x, *a, **k)[0])[0].tolist()
    assert w() == [0, 1, 2, 3, 4]
    assert w(top_k=2) == [1, 3] and w(top_k=3) == [0, 1, 3] and w(top_k=9) == [0, 1, 2, 3, 4]
    assert w(top_p=0.3) == [1] and w(top_p=0.65) == [1, 3] and w(top_p=0.75) == [0, 1, 3] and w(top_p=0.0) == [1]
    assert w(top_k=3, top_p=0.45) == [1] and w(top_k=3, top_p=0.51) == [1, 3]      # 0.4 of 0.8 is half
    assert w(min_p=0.5) == [1, 3] and w(min_p=2.0) == [1]
    assert w(0.0) == [1] and w(-1.0) == [1] and w(math.nan) == [1]
    assert np.allclose(O.sample(x, 0.5)[0] / O.sample(x, 0.5)[0].sum(), np.array([1, 16, 1, 9, 1]) / 28)
    assert O.sample(np.array([-math.inf, math.nan]))[0] is None
    assert O.sample(np.array([1.0, math.inf, math.nan, math.inf]))[0].tolist() == [0, 1, 0, 1]
    assert O.pick(np.array([0.0, 1, 0, 3]), 0.25)[0] == 3 and O.pick(np.array([0.0, 1, 0, 3]), 0.2)[0] == 1
    assert O.pick(np.array([1.0, 0]), 0.0)[0] == 0
