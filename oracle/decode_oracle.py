"""CPU oracle for the calls around the MLP: attention over a paged key/value cache, verification of
drafted trees, page operations.

TEST INFRASTRUCTURE ONLY, like dip_oracle.py: each definition taken step by step in 64 bits, entry by
entry and row by row, sharing no code with the HIP path.  Verification follows the rule as it is usually
stated (r <- norm((r - q)+) after each refused child), page operations work on Python lists.
"""
from __future__ import annotations

from typing import List, Optional, Sequence

import numpy as np


# ---- attention --------------------------------------------------------------------------------------
def ancestors(parents: Sequence[int]) -> List[Optional[List[int]]]:
    """For each node the list of its ancestors from the root down to itself, None if it is absent."""
    out: List[Optional[List[int]]] = []
    for t, up in enumerate(parents):
        if up == -1:
            out.append([t])
        elif 0 <= up < t and out[up] is not None:
            out.append(out[up] + [t])
        else:
            out.append(None)
    return out


def visible(n_before: int, rows: int, window: int, sinks: int, parents=None) -> np.ndarray:
    """bool [rows][n_before + rows]: which positions each row sees."""
    sees = np.zeros((rows, n_before + rows), dtype=bool)
    anc = ancestors(parents) if parents is not None else None
    for t in range(rows):
        if anc is not None and anc[t] is None:
            continue
        depth = t if anc is None else len(anc[t]) - 1
        pos = n_before + depth
        last = n_before + t if anc is None else n_before - 1
        for j in range(last + 1):
            sees[t, j] = window == 0 or j > pos - window or j < sinks
        if anc is not None:
            for a in anc[t]:
                sees[t, n_before + a] = True
    return sees


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, sees: np.ndarray, scale: float):
    """One entry: q [rows][Hq][D], k, v [keys][Hkv][D] (float64), sees [rows][keys].
    Returns (out, sum of p |v|, largest scale * sum |q k| of the visible keys), [rows][Hq][D] and [rows][Hq]."""
    rows, hq, d = q.shape
    group = hq // k.shape[1]
    out, mag = np.zeros((rows, hq, d)), np.zeros((rows, hq, d))
    big = np.zeros((rows, hq))
    for t in range(rows):
        at = np.nonzero(sees[t])[0]
        if at.size == 0:
            continue
        for h in range(hq):
            kk, vv = k[at, h // group], v[at, h // group]
            z = scale * (kk @ q[t, h])
            p = np.exp(z - z.max())
            p /= p.sum()
            out[t, h], mag[t, h] = p @ vv, p @ np.abs(vv)
            big[t, h] = scale * (np.abs(kk) @ np.abs(q[t, h])).max()
    return out, mag, big


# ---- verification -------------------------------------------------------------------------------------
def verify(parents, tokens, p: np.ndarray, q: np.ndarray, u, u_sample: float, max_kids: int):
    """One entry.  Returns (nodes that stand, next token)."""
    n = len(parents)
    if n == 0 or parents[0] != -1:
        return [], -1
    node, path = 0, [0]
    while True:
        r = p[node].astype(np.float64)
        qq = q[node].astype(np.float64)
        step = None
        for kid in [t for t in range(node + 1, n) if parents[t] == node][:max_kids]:
            x = tokens[kid]
            if 0 <= x < p.shape[1] and float(u[kid]) * qq[x] < r[x]:
                step = kid
                break
            r = np.maximum(r - qq, 0.0)
            if r.sum() > 0:
                r = r / r.sum()
        if step is None:
            break
        node = step
        path.append(node)
    if not r.sum() > 0:
        r = p[node].astype(np.float64)
    cum = np.cumsum(r)
    if not cum[-1] > 0:
        return path, -1
    over = np.nonzero(cum > float(u_sample) * cum[-1])[0]
    return path, int(over[0]) if over.size else int(np.nonzero(r > 0)[0][-1])


# ---- pages -----------------------------------------------------------------------------------------------
class Pool:
    """Tables, lengths and counts of a cache as lists, with the rows themselves in a dict by (page, slot).  Which
    entries of a step were granted nothing is remembered from reserve on: append and compact pass them over."""

    def __init__(self, n_pages: int, page: int, n_seqs: int, max_pages: int):
        self.page, self.max_pages = page, max_pages
        self.table = [[-1] * max_pages for _ in range(n_seqs)]
        self.len = [0] * n_seqs
        self.refs = [0] * n_pages
        self.rows = {}
        self.refused = set()

    def free(self, seqs):
        for s in seqs:
            if not 0 <= s < len(self.len):
                continue
            for j, pg in enumerate(self.table[s]):
                if pg >= 0:
                    self.refs[pg] -= 1
                self.table[s][j] = -1
            self.len[s] = 0

    def fork(self, src, dst):
        for a, b in zip(src, dst):
            for j in range(-(-self.len[a] // self.page)):
                self.table[b][j] = self.table[a][j]
                if self.table[b][j] >= 0:
                    self.refs[self.table[b][j]] += 1
            self.len[b] = self.len[a]

    def copy_pages(self, src, dst):
        for a, b in zip(src, dst):
            for s in range(self.page):
                if (a, s) in self.rows:
                    self.rows[b, s] = self.rows[a, s]

    def pages_of(self, s, n):
        """Places in the table that positions len .. len + n - 1 fall into."""
        return range(self.len[s] // self.page, -(-(self.len[s] + n) // self.page)) if n else range(0)

    def reserve(self, seqs, counts):
        free = [i for i, r in enumerate(self.refs) if r == 0]
        shared = [r > 1 for r in self.refs]
        asked, granted = 0, []
        for s, n in zip(seqs, counts):
            if self.len[s] + n > self.max_pages * self.page:
                granted.append(0)
                continue
            want = [j for j in self.pages_of(s, n) if self.table[s][j] < 0 or shared[self.table[s][j]]]
            ok = not want or asked + len(want) <= len(free)
            granted.append(int(ok))
            if ok:
                for i, j in enumerate(want):
                    new, old = free[asked + i], self.table[s][j]
                    if old >= 0:
                        self.refs[old] -= 1
                        for x in range(self.len[s] % self.page if j == self.len[s] // self.page else 0):
                            if (old, x) in self.rows:
                                self.rows[new, x] = self.rows[old, x]
                    self.refs[new] += 1
                    self.table[s][j] = new
            asked += len(want)
        # who is left alone with all its pages, the others having taken new ones, has its room too
        for i, (s, n) in enumerate(zip(seqs, counts)):
            if self.len[s] + n <= self.max_pages * self.page:
                if all(self.table[s][j] >= 0 and self.refs[self.table[s][j]] == 1 for j in self.pages_of(s, n)):
                    granted[i] = 1
        self.refused = {s for s, ok in zip(seqs, granted) if not ok}
        return granted

    def place(self, s, pos):
        j = pos // self.page
        pg = self.table[s][j] if j < self.max_pages else -1
        return (pg, pos % self.page) if pg >= 0 else None

    def append(self, seqs, rows):
        """rows: one list of row names per entry."""
        for s, names in zip(seqs, rows):
            for t, name in enumerate(names if s not in self.refused else []):
                self.rows[self.place(s, self.len[s] + t)] = name

    def compact(self, seqs, counts, paths, keep):
        for i, (s, n) in enumerate(zip(seqs, counts)):
            kept = min(max(keep[i], 0), n) if keep is not None else n
            if s in self.refused:
                kept = 0
            if paths is not None:
                for j in range(kept):
                    if j < paths[i][j] < n:
                        self.rows[self.place(s, self.len[s] + j)] = self.rows[self.place(s, self.len[s] + paths[i][j])]
            self.len[s] += kept
            for j in range(-(-self.len[s] // self.page), self.max_pages):
                if self.table[s][j] >= 0:
                    self.refs[self.table[s][j]] -= 1
                self.table[s][j] = -1


# ---- rows turned to their positions ------------------------------------------------------------------------
def turn(x: np.ndarray, positions, freq, interleaved: bool, scale: float = 1.0) -> np.ndarray:
    """x [rows][heads][dims] (float64): each pair a complex number, times scale * exp(i position freq)."""
    out, half = x.copy(), len(freq)
    first = 2 * np.arange(half) if interleaved else np.arange(half)
    second = first + (1 if interleaved else half)
    by = scale * np.exp(1j * np.asarray(positions, dtype=np.float64)[:, None] * np.asarray(freq)[None])
    z = (x[..., first] + 1j * x[..., second]) * by[:, None]
    out[..., first], out[..., second] = z.real, z.imag
    return out


def tree_positions(n_before: int, parents) -> List[int]:
    """Position of each node: as far behind the sequence as it is deep; an absent node's is the root's."""
    return [n_before + (len(a) - 1 if a else 0) for a in ancestors(parents)]


# ---- sampling ------------------------------------------------------------------------------------------------
def sample(logits: np.ndarray, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row: (kept weights by word, cuts one rule after the other over a sorted list; None if nothing is above -inf).
    The second result is the smallest distance, relative to the sum, of a weight sum or a weight from a rule's border."""
    x = np.where(np.isnan(logits), -np.inf, logits.astype(np.float64)) + 0.0
    out, close = np.zeros(len(x)), np.inf
    order = np.argsort(-x, kind="stable")
    order = order[x[order] > -np.inf]
    if not len(order):
        return None, close
    if not temperature > 0:
        out[order[0]] = 1.0
        return out, close
    top = x[order[0]]
    if top == np.inf:                                 # outweighs all that is finite, at any temperature
        w = (x[order] == top).astype(np.float64)
    else:
        with np.errstate(over="ignore"):
            w = np.exp((x[order] - top) / temperature)
    if top_k > 0:
        order, w = order[:top_k], w[:top_k]
    if top_p < 1:
        sums = np.cumsum(w)
        close = min(close, np.abs(sums[:-1] / sums[-1] - top_p).min(initial=np.inf))
        n = int(np.searchsorted(sums, top_p * sums[-1], side="left")) + 1
        order, w = order[:n], w[:n]
    if min_p > 0:
        edge = min(min_p, 1.0)
        close = min(close, np.abs(w[w != 1.0] / edge - 1).min(initial=np.inf))
        order, w = order[w >= edge], w[w >= edge]
    out[order] = w
    return out, close


def pick(weights: np.ndarray, u: float):
    """(the word at which the running sum passes u, its distance from a border relative to the sum)."""
    sums = np.cumsum(weights)
    over = np.nonzero(sums > u * sums[-1])[0]
    at = int(over[0]) if over.size else int(np.nonzero(weights)[0][-1])
    at_border = np.abs(sums / sums[-1] - u)[weights > 0]
    return at, float(at_border.min())


# ---- blocks of a long context ----------------------------------------------------------------------------------
def block_parts(n: int, page: int, block: int, sinks: int, recent: int):
    """(front, tail): positions [0, front) and [tail, n) are always read, blocks are chosen between."""
    tail = min(max(n - recent, 0), n - n % page) // block * block
    return min(-(-sinks // block) * block, tail), tail


def block_bounds(k: np.ndarray, most: float):
    """Keys of a block [positions][D] -> (lo, hi); NaN not counted, infinities as +-most, 0 where there is nothing."""
    lo, hi = np.zeros(k.shape[1]), np.zeros(k.shape[1])
    for d in range(k.shape[1]):
        x = k[:, d][~np.isnan(k[:, d])]
        if x.size:
            lo[d], hi[d] = max(min(x.min(), most), -most), max(min(x.max(), most), -most)
    return lo, hi


def choose_blocks(q: np.ndarray, lo: np.ndarray, hi: np.ndarray, first: int, n_select: int) -> List[int]:
    """q [heads of a group][D], lo and hi [blocks][D]: the numbers (from `first` on) of the chosen ones, ascending."""
    score = np.full(len(lo), -np.inf)
    for h in q:
        with np.errstate(invalid="ignore", over="ignore"):
            s = (np.maximum(h, 0) * hi + np.minimum(h, 0) * lo).sum(1)
        score = np.maximum(score, np.where(np.isnan(s), -np.inf, s))
    with np.errstate(over="ignore"):
        order = np.argsort(-score.astype(np.float32), kind="stable")[:n_select]
    return sorted(first + int(b) for b in order)


def block_visible(n: int, rows: int, front: int, tail: int, block: int, chosen, parents=None) -> np.ndarray:
    """bool [rows][n + rows]; chosen: the blocks of each row."""
    sees = visible(n, rows, 0, 0, parents)
    for t in range(rows):
        read = np.zeros(n + rows, dtype=bool)
        read[:front] = True
        read[tail:] = True
        for b in chosen[t]:
            read[b * block:(b + 1) * block] = True
        sees[t] &= read
    return sees
