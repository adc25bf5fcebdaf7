"""The page oracle on a pool that runs out, worked by hand: an entry that was granted nothing is neither written nor
committed, and what a sequence has committed is what its own steps put there."""
import random

from oracle import decode_oracle as O


def step(o, seqs, rows, paths=None, keep=None):
    granted = o.reserve(seqs, [len(r) for r in rows])
    o.append(seqs, rows)
    o.compact(seqs, [len(r) for r in rows], paths, keep)
    return granted


def held(o, s):
    """The rows that sequence s finds at its positions."""
    return [o.rows[o.place(s, i)] for i in range(o.len[s])]


def two_branches(pages, tail):
    """A prompt of four rows a page and `tail` more, forked, in a pool that has `pages` pages more."""
    o = O.Pool(2 + pages, 4, 3, 4)
    text = list("abcdefgh")[:4 + tail]
    assert step(o, [0], [text]) == [1]
    o.fork([0], [1])
    return o, text


def test_two_branches_of_a_shared_page_and_no_page_left():
    o, text = two_branches(0, 2)
    assert step(o, [0, 1], [["x"], ["y"]]) == [0, 0]
    assert o.len == [6, 6, 0] and o.refs == [2, 2] and held(o, 0) == held(o, 1) == text
    # and one after the other
    assert step(o, [1], [["y", "z"]]) == [0] and step(o, [0], [["x"]]) == [0]
    assert o.len == [6, 6, 0] and held(o, 0) == held(o, 1) == text


def test_who_is_left_alone_with_a_page_has_room_in_it():
    o, text = two_branches(1, 2)
    assert step(o, [0, 1], [["x"], ["y", "z"]]) == [1, 1]       # 0 takes the free page, the old one is 1's alone
    assert o.refs == [2, 1, 1] and o.table[0][:2] == [0, 2] and o.table[1][:2] == [0, 1]
    assert held(o, 0) == text + ["x"] and held(o, 1) == text + ["y", "z"]
    o, text = two_branches(1, 2)
    assert step(o, [0, 1], [["x"], ["y", "z", "u"]]) == [1, 0]  # 1 would need another one
    assert o.len == [7, 6, 0] and held(o, 0) == text + ["x"] and held(o, 1) == text


def test_a_kept_path_that_leads_past_the_last_page():
    o, text = O.Pool(2, 4, 1, 4), list("abcdef")
    step(o, [0], [text])
    assert step(o, [0], [list("stuvwx")], [[0, 5]], [2]) == [0]
    assert o.len == [6] and held(o, 0) == text


def test_rows_behind_the_table():
    o = O.Pool(9, 4, 1, 2)
    step(o, [0], [list("abcdef")])
    assert step(o, [0], [list("xyz")]) == [0]                   # two of them would have had a place
    assert o.len == [6] and held(o, 0) == list("abcdef")


def test_any_order_of_calls_keeps_every_sequence_to_itself():
    for seed in range(200):
        rng = random.Random(seed)
        page, n = rng.choice([1, 2, 4, 8]), 5
        o = O.Pool(rng.randint(4, 14), page, n, rng.randint(3, 9))
        text, name = [[] for _ in range(n)], 0
        for _ in range(25):
            what = rng.random()
            if what < 0.2:
                s = rng.sample(range(n), rng.randint(1, 2))
                o.free(s)
                for x in s:
                    text[x] = []
            elif what < 0.45:
                empty, full = [s for s in range(n) if not text[s]], [s for s in range(n) if text[s]]
                if empty and full:
                    dst = rng.sample(empty, rng.randint(1, len(empty)))
                    src = [rng.choice(full) for _ in dst]
                    o.fork(src, dst)
                    for a, b in zip(src, dst):
                        text[b] = list(text[a])
            else:
                seqs = rng.sample(range(n), rng.randint(1, n))
                rows = []
                for _ in seqs:
                    r = rng.choice([0, 1, 1, 2, 3, 7])
                    rows.append(list(range(name, name + r)))
                    name += r
                paths = [sorted(rng.sample(range(len(r)), rng.randint(0, len(r)))) for r in rows]
                for s, r, p, ok in zip(seqs, rows, paths, step(o, seqs, rows, paths, [len(p) for p in paths])):
                    if ok:
                        text[s] += [r[i] for i in p]
            assert o.len == [len(t) for t in text]
            assert [held(o, s) for s in range(n)] == text
            named = [pg for t in o.table for pg in t if pg >= 0]
            assert o.refs == [named.count(i) for i in range(len(o.refs))]
