"""Steps in a pool that runs out: an entry that was granted nothing is neither written nor committed, in any layer, and
what a sequence finds at its positions is what its own steps put there."""
import random

import pytest
import torch

from test_gpu_decode import Paged

pytestmark = pytest.mark.gpu


class Text(Paged):
    """Paged with a list of each sequence's rows, kept from the steps alone."""

    def __init__(self, *a, **kw):
        super().__init__(*a, **kw)
        self.text = [[] for _ in self.o.len]

    def step(self, seqs, counts, paths=None, keep=None):
        first = self.next
        super().step(seqs, counts, paths, keep)
        for i, (s, n) in enumerate(zip(seqs, counts)):
            names = list(range(first + sum(counts[:i]), first + sum(counts[:i]) + n))
            if s not in self.o.refused:
                kept = n if keep is None else min(max(keep[i], 0), n)
                self.text[s] += [names[paths[i][j]] for j in range(kept)] if paths else names[:kept]
        self.read()

    def free(self, seqs):
        super().free(seqs)
        for s in seqs:
            self.text[s] = []
        self.read()

    def fork(self, src, dst):
        super().fork(src, dst)
        for a, b in zip(src, dst):
            self.text[b] = list(self.text[a])
        self.read()

    def read(self):
        assert self.c.seq_len.tolist() == [len(t) for t in self.text]
        page = self.c.k.shape[3]
        for s, names in enumerate(self.text):
            if not names:
                continue
            at = torch.arange(len(names), device="cuda")
            pg, sl = self.c.page_table[s][at // page].long(), at % page
            want = torch.tensor(names, device="cuda")[:, None] + 1000 * torch.arange(self.layers, device="cuda")
            for t, sign in ((self.c.k, 1), (self.c.v, -1)):
                assert (t[:, pg, :, sl] == sign * want[:, :, None, None]).all(), s


def branches(pages, tail, **kw):
    """A prompt of a page of four rows and `tail` more, forked, in a pool that has `pages` pages more."""
    c = Text(n_pages=2 + pages, page=4, n_seqs=3, max_pages=4, **kw)
    c.step([0], [4 + tail])
    c.fork([0], [1])
    return c


@pytest.mark.parametrize("slot_major", [False, True])
def test_two_branches_of_a_shared_page_and_no_page_left(slot_major):
    c = branches(0, 2, slot_major=slot_major)
    c.step([0, 1], [1, 2])
    c.step([1], [2], [[1]], [1])
    c.step([0], [1])
    assert c.o.len == [6, 6, 0]
    c.free([0])                                      # now the tail is the other's alone
    c.step([1], [2])
    assert c.o.len == [0, 8, 0]


def test_who_is_left_alone_with_a_page_has_room_in_it():
    c = branches(1, 2)
    c.step([0, 1], [1, 2])
    assert c.o.len == [7, 8, 0] and c.o.refs == [2, 1, 1]
    c = branches(1, 2)
    c.step([0, 1], [1, 3])                           # one row more than the page has left
    assert c.o.len == [7, 6, 0]
    c.step([1], [2])
    assert c.o.len == [7, 8, 0]


def test_a_kept_path_that_leads_past_the_last_page():
    c = Text(n_pages=2, page=4, n_seqs=1, max_pages=4)
    c.step([0], [6])
    c.step([0], [6], [[0, 5]], [2])
    assert c.o.len == [6]
    c.step([0], [2], [[0, 1]], [2])
    assert c.o.len == [8]


def test_rows_behind_the_table():
    c = Text(n_pages=9, page=4, n_seqs=2, max_pages=2)
    c.step([0, 1], [6, 3])
    c.step([0, 1], [3, 5])                           # too long by one; just as long as it may be
    assert c.o.len == [6, 8]
    c.step([0, 1], [2, 1], [[0, 1], [0]], [2, 1])
    assert c.o.len == [8, 8]


def test_many_entries_and_few_pages():
    c = Text(n_pages=1500, page=2, n_seqs=1024, max_pages=12, hkv=1, layers=1)
    rng = random.Random(1)
    c.step(list(range(400)), [rng.randint(0, 5) for _ in range(400)])
    held = [s for s in range(400) if c.text[s]][:300]
    c.fork(held, list(range(400, 400 + len(held))))
    for _ in range(2):
        live = rng.sample(range(1024), 900)
        c.step(live, [rng.randint(0, 4) for _ in live])


@pytest.mark.parametrize("seed", range(24))
def test_any_order_of_calls_keeps_every_sequence_to_itself(seed):
    rng = random.Random(seed)
    page, n = rng.choice([1, 2, 4, 8]), 5
    c = Text(n_pages=rng.randint(4, 14), page=page, n_seqs=n, max_pages=rng.randint(3, 9), hkv=rng.choice([1, 3]), layers=2,
             slot_major=rng.random() < 0.5)
    for _ in range(14):
        what = rng.random()
        empty, full = [s for s in range(n) if not c.text[s]], [s for s in range(n) if c.text[s]]
        if what < 0.2:
            c.free(rng.sample(range(n), rng.randint(1, 2)))
        elif what < 0.45 and empty and full:
            dst = rng.sample(empty, rng.randint(1, len(empty)))
            c.fork([rng.choice(full) for _ in dst], dst)
        else:
            seqs = rng.sample(range(n), rng.randint(1, n))
            counts = [rng.choice([0, 1, 1, 2, 3, 7]) for _ in seqs]
            paths = [sorted(rng.sample(range(r), rng.randint(0, r))) for r in counts]
            c.step(seqs, counts, paths, [len(p) for p in paths])
