"""Batches that mix single tokens with pieces of prompts, and verification of rows that take several passes of a
workgroup."""
import numpy as np
import pytest
import torch

from test_gpu_decode import Setup, check_verify, random_tree, verify_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(64, 1), (96, 16), (128, 64)])
def test_single_tokens_beside_a_piece_of_a_prompt(dtype, d, page):
    lens = [1700, 0, 300, 31, 2600, 64] + [7 * i for i in range(20)]
    rows = [1, 150, 1, 3, 1, 70] + [1] * 20
    s = Setup(dtype, lens, rows, 8, 2, d, page, slot_major=page == 16, seed=d)
    for window, sinks in [(0, 0), (100, 4), (1000, 70)]:
        s.check(s.run(window, sinks), window, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_small_and_wide_trees_in_one_batch(dtype):
    lens, rows = [900, 2000, 5, 130], [1, 64, 8, 33]
    s = Setup(dtype, lens, rows, 8, 2, 128, 16, seed=1)
    par = [random_tree(np.random.default_rng(2), n, absent=n == 33) for n in rows]
    for window, sinks in [(0, 0), (500, 3)]:
        s.check(s.run(window, sinks, par), window, sinks, par)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_verify_with_two_passes_to_a_chunk(dtype):
    # more chunks of 4096 words than workgroups fit the chip at a time: chunks of 8192
    rng = np.random.default_rng(3)
    trees = [random_tree(rng, int(n), kids=2) for n in rng.integers(1, 5, 36)]
    p, q, tokens, u, us = verify_inputs(rng, trees, 126001, dtype=dtype)
    check_verify(trees, p, q, tokens, u, us, 3)
    us[::2], us[1::2] = 0.0, np.nextafter(np.float32(1), np.float32(0))
    check_verify(trees, p, q, tokens, u, us, 3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [262145, 300007, 600000])
def test_verify_vocabularies_beyond_one_pass_of_all_chunks(vocab, dtype):
    rng = np.random.default_rng(vocab)
    trees = [random_tree(rng, n, kids=3) for n in (1, 4, 6)]
    p, q, tokens, u, us = verify_inputs(rng, trees, vocab, near=1.5, dtype=dtype)
    check_verify(trees, p, q, tokens, u, us, 63)
    check_verify(trees, p, q, tokens, u, np.full(3, 0.9999999, np.float32), 63)
