"""What is timed when the operators of a speculative decode step are looked at: attention over a
paged key/value cache (a sliding window with sinks; a tree of drafted tokens), the verification of
the drafts against the target's probabilities, and the cache's page operations.

A case is a dict of plain values:
  op      "window", "tree", "verify" or "pages"
  dtype   "bf16" or "f32": the cache, queries and outputs (verify: the probabilities)
  B       batch entries;   T  most rows of an entry (prompt tokens, tree nodes)
  L       most tokens that an entry has in the cache before its rows
  Hq, Hkv, D   query heads, key/value heads, head dimension
  page    slots of a page;   slot_major  the cache stores [page][slot][head], else [page][head][slot]
  window, sinks   what a row sees of its past (window 0: all of it)
  V, kids vocabulary, most children of a tree node
  layers, fan     pages: layers of the cache, branches forked from one sequence
  ragged  entries differ in length and rows
Where `own` is false, run() computes the plain form; where it is true, it calls the package.
"""
import math

import torch

own = False

GOLD = 0.6180339887498949


def listed():
    return [
        # the smallest call of a decode loop: one token each for two short chats
        dict(name="window decode 2x700", op="window", dtype="bf16", B=2, T=1, L=700, Hq=32, Hkv=8, D=128, page=16,
             slot_major=False, window=1024, sinks=4, ragged=True),
        # a serving batch of single tokens far into their contexts: the window bounds what is read
        dict(name="window decode 32x12k", op="window", dtype="bf16", B=32, T=1, L=12000, Hq=40, Hkv=10, D=128, page=16,
             slot_major=False, window=2047, sinks=4, ragged=True),
        # pieces of prompts in full precision, odd lengths, a head dimension of 96, slots before heads
        dict(name="window prompt f32 3x777", op="window", dtype="f32", B=3, T=777, L=401, Hq=32, Hkv=32, D=96, page=64,
             slot_major=True, window=256, sinks=1, ragged=True),
        # the second half of a long prompt beside a shorter one: bound by the matrix cores
        dict(name="window prompt 2x4096", op="window", dtype="bf16", B=2, T=4096, L=4096, Hq=40, Hkv=10, D=128, page=32,
             slot_major=False, window=2047, sinks=4, ragged=True),
        # a tree of seven drafts for each of three short sequences in full precision, every head its own cache
        dict(name="tree f32 3x7 over 1500", op="tree", dtype="f32", B=3, T=7, L=1500, Hq=32, Hkv=32, D=96, page=32,
             slot_major=True, window=512, sinks=2, kids=3, ragged=True),
        # the batch that the pruned layers take in one call: eight nodes, eight sequences
        dict(name="tree 8x8 over 8k", op="tree", dtype="bf16", B=8, T=8, L=8192, Hq=32, Hkv=8, D=128, page=16,
             slot_major=False, window=0, sinks=0, kids=2, ragged=True),
        # wide trees over long documents
        dict(name="tree 4x64 over 48k", op="tree", dtype="bf16", B=4, T=64, L=49152, Hq=40, Hkv=10, D=128, page=64,
             slot_major=False, window=0, sinks=0, kids=4, ragged=True),
        # one sequence, a chain of four drafts, a small vocabulary
        dict(name="verify chain 1x5 of 32064", op="verify", dtype="f32", B=1, T=5, V=32064, kids=1, ragged=False),
        # trees of a batch, probabilities kept in 16 bits
        dict(name="verify tree 16x8 bf16", op="verify", dtype="bf16", B=16, T=8, V=128256, kids=3, ragged=True),
        # a large batch of trees over a large vocabulary
        dict(name="verify tree 64x16 of 128256", op="verify", dtype="f32", B=64, T=16, V=128256, kids=2, ragged=True),
        # branches of two chats: a few drafts each, most of them dropped
        dict(name="pages 6 branches of 2", op="pages", dtype="bf16", B=6, T=8, L=300, Hkv=8, D=128, page=16, layers=32,
             slot_major=False, fan=3, ragged=True),
        # continuations of shared prompts, 256 rows each
        dict(name="pages 16 branches of 4", op="pages", dtype="bf16", B=16, T=256, L=1900, Hkv=10, D=128, page=64, layers=40,
             slot_major=True, fan=4, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _most(op, key):
    return max(work(c)[key] for c in listed() if c["op"] == op)


def draw(rng):
    op = rng.choice(["window", "tree", "verify", "pages"])
    while True:
        c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "f32"]), ragged=rng.random() < 0.7)
        if op == "verify":
            c.update(B=_log(rng, 1, 64), T=rng.randint(1, 16), V=_log(rng, 1000, 128256), kids=rng.randint(1, 4))
        else:
            c.update(page=rng.choice([8, 16, 32, 64, 128]), slot_major=rng.random() < 0.4, D=rng.choice([64, 96, 128, 128]),
                     Hkv=rng.choice([1, 2, 4, 8, 8, 10, 16, 32]))
            if op == "pages":
                c.update(B=_log(rng, 1, 16), T=_log(rng, 1, 256), L=_log(rng, 1, 1900), layers=_log(rng, 1, 40), fan=rng.randint(1, 4))
            else:
                c["Hq"] = c["Hkv"] * rng.choice([1, 2, 3, 4, 5, 7, 8])
                c["window"], c["sinks"] = (_log(rng, 64, 4096), rng.randint(0, 8)) if rng.random() < 0.6 else (0, 0)
                if op == "tree":
                    c.update(B=_log(rng, 1, 16), T=_log(rng, 1, 64), L=_log(rng, 1, 49152), kids=rng.randint(1, 4))
                elif rng.random() < 0.5:
                    c.update(B=_log(rng, 1, 32), T=1, L=_log(rng, 1, 12000))
                else:
                    c.update(B=_log(rng, 1, 4), T=_log(rng, 2, 4096), L=_log(rng, 1, 4096))
        w = work(c)
        if w["bytes"] > _most(op, "bytes") or w["flops"] > _most(op, "flops"):
            continue
        if op in ("window", "tree") and c["B"] * c["Hq"] * c["T"] * (c["L"] + c["T"]) > 2 * 40 * 4096 * 8192:
            continue                                  # (the plain form's scores)
        if op != "verify" and c.get("layers", 1) * _n_pages(c) * c["page"] * c["Hkv"] * c["D"] > 1 << 31:
            continue
        return c


# ---- the entries of a case: fixed by the case alone, so that work() knows them --------------------
def _lens(c):
    """Tokens of each sequence in the cache; the first has L."""
    n = c["B"] if c["op"] != "pages" else -(-c["B"] // c["fan"])
    return [c["L"] if i == 0 or not c["ragged"] else max(1, int(c["L"] * (1 - 0.9 * ((i * GOLD) % 1.0)))) for i in range(n)]


def _rows(c):
    """Rows of each entry; the first has T."""
    return [c["T"] if i == 0 or not c["ragged"] else max(1, int(c["T"] * (1 - 0.7 * ((i * GOLD * GOLD) % 1.0)))) for i in range(c["B"])]


def _keeps(c):
    """Rows of each entry that are kept (pages): all drafts of some, few of others."""
    return [max(1, int(r * (1 - ((i * GOLD) % 1.0)))) for i, r in enumerate(_rows(c))]


def _need(c):
    """Pages that each entry may come to hold."""
    lens = _lens(c)
    return [-(-(lens[i // c.get("fan", 1) if c["op"] == "pages" else i] + r) // c["page"]) for i, r in enumerate(_rows(c))]


def _n_pages(c):
    spare = sum(-(-n // c["page"]) for n in _lens(c)) if c["op"] == "pages" else 0
    return sum(_need(c)) + spare + 7


def _parents(c):
    """Parent of each node, per entry: node 0 is the last committed token, nobody has more than `kids` children."""
    out = []
    for e, n in enumerate(_rows(c)):
        par, kids = [-1], [0]
        for t in range(1, n):
            at = int((((t + 3 * e) * GOLD) % 1.0) * t)
            while kids[at] >= c["kids"]:
                at = (at + 1) % t
            kids[at] += 1
            par.append(at)
            kids.append(0)
        out.append(par)
    return out


def _depths(par):
    d = []
    for p in par:
        d.append(0 if p < 0 else d[p] + 1)
    return d


def _seen(c, n, rows):
    """(visible pairs, keys that any row sees) of one entry with n tokens before its rows."""
    w, s = c["window"] or (1 << 60), c["sinks"]
    pairs, first = 0, 1 << 60
    for pos in rows:
        lo = max(0, pos - w + 1)
        pairs += pos + 1 - lo + min(s, lo)
        first = min(first, lo)
    return pairs, max(rows) + 1 - first + min(s, first)


def work(c):
    es = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "verify":                           # the two rows that the walk ends at
        return {"bytes": sum(2 * c["V"] * es for _ in _rows(c)) + 16 * sum(_rows(c)), "flops": 4 * c["V"] * c["B"]}
    if c["op"] == "pages":
        row = c["layers"] * c["Hkv"] * c["D"] * 2 * es
        lens = _lens(c)
        tail = sum(lens[i // c["fan"]] % c["page"] for i in range(c["B"]))
        moved = sum(_keeps(c)) - c["B"]
        table = 4 * (_n_pages(c) + 4 * sum(_need(c)))
        return {"bytes": 2 * row * (tail + sum(_rows(c)) + max(0, moved)) + table, "flops": 1}
    pairs = keys = rows = 0
    for i, (n, r) in enumerate(zip(_lens(c), _rows(c))):
        if c["op"] == "window":
            a, b = _seen(c, n, [n + t for t in range(r)])
        else:                                         # a node sees its ancestors, one of each depth
            a, b = _seen(c, n, [n + d for d in _depths(_parents(c)[i])])
            b += r - 1 - max(_depths(_parents(c)[i]))
        pairs, keys, rows = pairs + a, keys + b, rows + r
    return {"bytes": es * c["D"] * (2 * keys * c["Hkv"] + 2 * rows * c["Hq"]), "flops": 4 * c["D"] * c["Hq"] * pairs}


# ---- inputs ---------------------------------------------------------------------------------------
def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _starts(rows):
    s = [0]
    for r in rows:
        s.append(s[-1] + r)
    return _ints(s)


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    rows = _rows(c)
    n = sum(rows)
    s = {"case": c, "row_start": _starts(rows), "n_rows": n, "max_rows": max(rows)}
    if c["op"] in ("tree", "verify"):
        s["parents"] = _ints([p for par in _parents(c) for p in par])
    if c["op"] == "verify":
        logits = 2.5 * normal(n, c["V"])              # a peaked target and a draft that follows it
        s["p"] = torch.softmax(logits, -1).to(dt)
        s["q"] = torch.softmax(0.9 * logits + 0.6 * normal(n, c["V"]), -1).to(dt)
        at = torch.where(s["parents"] >= 0, s["parents"], 0) + torch.repeat_interleave(s["row_start"][:-1], torch.diff(s["row_start"]).long(), output_size=n)
        drawn = torch.multinomial(s["q"].float(), c["kids"], replacement=True, generator=g)
        which = torch.randint(0, c["kids"], (n,), generator=g, device="cuda")
        s["tokens"] = drawn[at.long(), which].to(torch.int32)
        s["u"] = torch.rand(n, generator=g, device="cuda")
        s["u_sample"] = torch.rand(c["B"], generator=g, device="cuda")
        return s
    # a cache whose pages lie scattered, as after hours of serving
    lens, need, P, H, D = _lens(c), _need(c), _n_pages(c), c["Hkv"], c["D"]
    seqs_n = len(lens) + (c["B"] if c["op"] == "pages" else 0)
    max_pages = max(need)
    order = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
    table = torch.full((seqs_n, max_pages), -1, dtype=torch.int32, device="cuda")
    refs = torch.zeros(P, dtype=torch.int32, device="cuda")
    used = 0
    for i, ln in enumerate(lens):
        k = -(-ln // c["page"]) if c["op"] == "pages" else need[i]
        table[i, :k] = order[used:used + k]
        used += k
    refs[order[:used].long()] = 1
    shape = (c.get("layers", 1), P, c["page"], H, D) if c["slot_major"] else (c.get("layers", 1), P, H, c["page"], D)
    wide = torch.exp(0.4 * normal(D))                 # keys have a few loud channels
    raw = lambda f: torch.empty(shape, dtype=dt, device="cuda").normal_(generator=g).mul_(f)
    k, v = raw(wide.to(dt)), raw(1.0)
    if c["slot_major"]:
        k, v = k.transpose(2, 3), v.transpose(2, 3)
    s.update(k=k, v=v, table=table, refs=refs, max_len=max(ln + r for ln, r in zip(lens, rows)) if c["op"] != "pages" else c["L"] + c["T"],
             seq_len=_ints(lens + [0] * (seqs_n - len(lens))))
    if c["op"] == "pages":
        s["dst"] = torch.arange(len(lens), seqs_n, dtype=torch.int32, device="cuda")
        s["src"] = torch.arange(c["B"], dtype=torch.int32, device="cuda") // c["fan"]
        s["seqs"] = s["dst"]
        s["new_k"], s["new_v"] = normal(c["layers"], n, H, D).to(dt), normal(c["layers"], n, H, D).to(dt)
        s["keep"] = _ints(_keeps(c))
        path = torch.full((n,), -1, dtype=torch.int32, device="cuda")
        at = 0
        for r, m in zip(rows, _keeps(c)):             # a root and an ascending choice of the others
            pick = torch.randperm(r - 1, generator=g, device="cuda")[:m - 1].sort().values + 1
            path[at] = 0
            path[at + 1:at + m] = pick.to(torch.int32)
            at += r
        s["path"] = path
    else:
        s["seqs"] = torch.arange(c["B"], dtype=torch.int32, device="cuda")
        s["q"] = (1.5 * normal(n, c["Hq"], D)).to(dt)
    return s


# ---- the package's calls ----------------------------------------------------------------------------
def _handles(s):
    """What a program keeps beside its data: descriptors, output buffers, workspace."""
    import paper_2412_01380_amd as A
    c = s["case"]
    h = {"A": A, "batch": A.Batch(s["row_start"], s["n_rows"], s["max_rows"], seqs=s.get("seqs"), max_len=s.get("max_len", 0))}
    ints = lambda m: torch.empty(m, dtype=torch.int32, device="cuda")
    if c["op"] == "verify":
        h.update(keep=ints(c["B"]), path=ints(s["n_rows"]), token=ints(c["B"]))
        size = A.dip_verify_tree_workspace_bytes(h["batch"], c["V"], c["kids"])
    else:
        h["cache"] = A.KvCache(s["k"], s["v"], s["table"], s["seq_len"], s["refs"])
        if c["op"] == "pages":
            h["granted"] = ints(c["B"])
            size = A.dip_kv_reserve_workspace_bytes(h["cache"], h["batch"])
        else:
            h["out"] = torch.empty_like(s["q"])
            size = A.dip_attention_workspace_bytes(h["cache"], h["batch"], c["Hq"], c["window"], c["sinks"])
    h["ws"] = torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")
    return h


def _call(s):
    if "handles" not in s:
        s["handles"] = _handles(s)
    c, h = s["case"], s["handles"]
    A, b = h["A"], h["batch"]
    if c["op"] == "verify":
        A.dip_verify_tree(b, s["tokens"], s["parents"], s["p"], s["q"], s["u"], s["u_sample"], c["kids"], h["keep"], h["path"],
                          h["token"], h["ws"])
        return h["keep"], h["path"], h["token"]
    if c["op"] == "pages":
        A.dip_kv_free(h["cache"], s["dst"])
        A.dip_kv_fork(h["cache"], s["src"], s["dst"])
        A.dip_kv_reserve(h["cache"], b, h["granted"], h["ws"])
        A.dip_kv_append(h["cache"], 0, b, s["new_k"], s["new_v"])
        A.dip_kv_compact(h["cache"], b, s["path"], s["keep"])
        return s["k"], s["v"], s["table"], s["seq_len"], s["refs"], h["granted"]
    if c["op"] == "window":
        A.dip_window_attention(h["cache"], 0, b, s["q"], 1 / math.sqrt(c["D"]), c["window"], c["sinks"], h["out"], h["ws"])
    else:
        A.dip_tree_attention(h["cache"], 0, b, s["parents"], s["q"], 1 / math.sqrt(c["D"]), c["window"], c["sinks"], h["out"], h["ws"])
    return h["out"]


def run(s):
    if own:
        return _call(s)
    return {"window": _attend, "tree": _attend, "verify": _verify, "pages": _pages}[s["case"]["op"]](s)


# ---- the plain forms ------------------------------------------------------------------------------------
def _of_rows(s):
    """(entry, place in it) of each row."""
    at = torch.arange(s["n_rows"], device="cuda")
    b = torch.searchsorted(s["row_start"][1:].long(), at, right=True)
    return b, at - s["row_start"][b]


def _ancestors(parents, b, t, entries, most):
    """[entries, most, most]: whether a node is another's ancestor, or itself."""
    step = torch.zeros(entries, most, most, device="cuda")
    step[b, t, parents.clamp(min=0).long()] = (parents >= 0).float()
    eye = torch.eye(most, device="cuda")
    return torch.linalg.matrix_power(eye + step, max(1, most - 1)) > 0


def _attend(s):
    c = s["case"]
    B, T, Hq, H, D = c["B"], s["max_rows"], c["Hq"], c["Hkv"], c["D"]
    b, t = _of_rows(s)
    pages = s["table"][s["seqs"].long()].clamp(min=0).long()
    # [B, H, keys, D], every page that a sequence has a place for
    k = s["k"][0][pages].transpose(1, 2).reshape(B, H, -1, D).float()
    v = s["v"][0][pages].transpose(1, 2).reshape(B, H, -1, D).float()
    q = torch.zeros(B, T, Hq, D, device="cuda")
    q[b, t] = s["q"].float()
    q = q.view(B, T, H, Hq // H, D).permute(0, 2, 3, 1, 4).reshape(B, H, -1, D)
    n = s["seq_len"][s["seqs"].long()].view(B, 1, 1).long()
    j = torch.arange(k.shape[2], device="cuda").view(1, 1, -1)
    if c["op"] == "tree":
        anc = _ancestors(s["parents"], b, t, B, T)
        pos = n + anc.sum(-1, keepdim=True) - 1
        inside = torch.gather(anc, 2, (j - n).clamp(0, T - 1).expand(B, T, -1)) & (j >= n) & (j < n + T)
        sees = (j < n) | inside
    else:
        pos = n + torch.arange(T, device="cuda").view(1, T, 1)
        sees, inside = j <= pos, torch.zeros_like(j <= pos)
    if c["window"]:
        sees = sees & ((j > pos - c["window"]) | (j < c["sinks"]) | inside)
    z = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(D)
    z = z.view(B, H, Hq // H, T, -1).masked_fill_(~sees[:, None, None], -math.inf)
    z = torch.exp(z - z.amax(-1, keepdim=True))
    z = (z / z.sum(-1, keepdim=True)).view(B, H, -1, k.shape[2])
    o = torch.matmul(z, v).view(B, H, Hq // H, T, D).permute(0, 3, 1, 2, 4).reshape(B, T, Hq, D)
    return o[b, t].to(s["q"].dtype)


def _verify(s):
    """Child j of a node (in order) is taken where u q(x) G_j < (p(x) - lam_j q(x))+, with lam_0 = 0, G_0 = 1,
    lam_(j+1) = lam_j + G_j, G_j = sum (p - lam_j q)+; the next token is drawn from (p - lam_m q)+ of the last node
    that was taken, m its children.  Decisions have to be the same ones, so sums are kept in 64 bits."""
    c, n = s["case"], s["n_rows"]
    B, T = c["B"], s["max_rows"]
    b, t = _of_rows(s)
    first = s["row_start"][:-1].long()
    par = s["parents"].long()
    up = torch.where(par >= 0, par, 0) + first[b]     # the parent's row
    p, q = s["p"].double(), s["q"].double()
    sibling = (b[:, None] == b[None]) & (par[:, None] == par[None]) & (par[:, None] >= 0)
    order = (sibling & (t[None] < t[:, None])).sum(1)          # earlier children of the same node
    kids = ((b[:, None] == b[None]) & (par[None] == t[:, None])).sum(1)
    lam, G = torch.zeros(n, c["kids"] + 1, device="cuda", dtype=torch.float64), torch.ones(n, c["kids"] + 1, device="cuda", dtype=torch.float64)
    for j in range(c["kids"]):
        lam[:, j + 1] = lam[:, j] + G[:, j]
        G[:, j + 1] = (p - lam[:, j + 1, None] * q).clamp_(min=0).sum(1)
    x = s["tokens"].long()
    left = (p[up, x] - lam[up, order] * q[up, x]).clamp(min=0)
    passed = (s["u"].double() * q[up, x] * G[up, order] < left) & (par >= 0)
    earlier = sibling & (t[None] < t[:, None]) & passed[None]
    taken = torch.zeros(B, T, device="cuda")
    taken[b, t] = ((passed & ~earlier.any(1)) | (t == 0)).float()
    there = torch.zeros(B, T, device="cuda", dtype=torch.bool)
    there[b, t] = True
    anc = _ancestors(s["parents"], b, t, B, T)
    on = (torch.matmul(anc.float(), 1 - taken[:, :, None])[:, :, 0] == 0) & there
    keep = on.sum(1)
    place = torch.cumsum(on, 1) - 1
    path = torch.full((n + 1,), -1, dtype=torch.int32, device="cuda")
    path[torch.where(on, first[:, None] + place, n).view(-1)] = torch.arange(T, device="cuda", dtype=torch.int32).expand(B, T).reshape(-1)
    path[n] = -1
    last = first + torch.where(on, torch.arange(T, device="cuda"), -1).amax(1)
    m = kids[last]
    r = (p[last] - lam[last, m, None] * q[last]).clamp_(min=0)
    r = torch.where(r.sum(1, keepdim=True) > 0, r, p[last])
    run_sum = torch.cumsum(r, 1)
    above = run_sum > s["u_sample"].double()[:, None] * run_sum[:, -1:]
    token = torch.where(above.any(1), above.int().argmax(1), (r > 0).int().cumsum(1).argmax(1))
    return keep.to(torch.int32), path[:n].contiguous(), token.to(torch.int32)


def _pages(s):
    """Frees the branches, forks them again, makes room for their rows, writes these, keeps the path."""
    c = s["case"]
    page, table, refs, size, k, v = c["page"], s["table"], s["refs"], s["seq_len"], s["k"], s["v"]
    dst, src = s["dst"].long(), s["src"].long()
    j = torch.arange(table.shape[1], device="cuda")
    count = lambda of, sign: refs.index_add_(0, of.clamp(min=0).view(-1).long(), sign * (of >= 0).view(-1).int())
    count(table[dst], -1)
    table[dst] = -1
    size[dst] = 0
    held = (size[src] + page - 1) // page
    table[dst] = torch.where(j[None] < held[:, None], table[src], -1)
    count(table[dst], 1)
    size[dst] = size[src]
    # room for the rows: the lowest free pages, in order; a shared last page is copied
    rows = torch.diff(s["row_start"])
    n = size[dst]
    mine = table[dst]
    wanted = (j[None] >= (n // page)[:, None]) & (j[None] < ((n + rows + page - 1) // page)[:, None])
    wanted &= (mine < 0) | (refs[mine.clamp(min=0).long()] > 1)
    free = torch.argsort((refs != 0).int(), stable=True)
    total = torch.cumsum(wanted.sum(1), 0)
    granted = (wanted.sum(1) == 0) | (total <= (refs == 0).sum())
    rank = (torch.cumsum(wanted.view(-1), 0) - 1).view_as(wanted)
    wanted &= granted[:, None]
    fresh = torch.where(wanted, free[rank.clamp(0, free.shape[0] - 1)].int(), mine)
    at = (n // page).clamp(max=table.shape[1] - 1).long()[:, None]
    old, new = mine.gather(1, at)[:, 0], fresh.gather(1, at)[:, 0]
    tail = torch.where((old != new) & (old >= 0), n % page, 0)
    some = (tail > 0).int().argmax()                  # (entries without a copy repeat one that has it)
    old, new, tail = (torch.where(tail > 0, a, a[some]) for a in (old, new, tail))
    part = (torch.arange(page, device="cuda")[None] < tail[:, None])[None, :, None, :, None]
    old, new = old.clamp(min=0).long(), new.clamp(min=0).long()
    put = torch.where(tail > 0, new, old)
    k[:, put] = torch.where(part, k[:, old], k[:, put])
    v[:, put] = torch.where(part, v[:, old], v[:, put])
    count(torch.where(wanted, mine, -1), -1)
    count(torch.where(wanted, fresh, -1), 1)
    table[dst] = fresh
    # the rows, then those of the path moved to the front
    b, t = _of_rows(s)
    place = n[b] + t
    where = fresh[b, place // page].long()
    k[:, where, :, place % page] = s["new_k"].transpose(0, 1)
    v[:, where, :, place % page] = s["new_v"].transpose(0, 1)
    kept = t < s["keep"][b]
    pick = n[b] + torch.where(kept, s["path"], t)
    from_page = fresh[b, pick // page].long()
    k[:, where, :, place % page] = k[:, from_page, :, pick % page]
    v[:, where, :, place % page] = v[:, from_page, :, pick % page]
    size[dst] = n + s["keep"]
    over = j[None] >= ((size[dst] + page - 1) // page)[:, None]
    count(torch.where(over, fresh, -1), -1)
    table[dst] = torch.where(over, -1, fresh)
    return k, v, table, size, refs, granted.int()


# ---- the definitions in 64 bits, entry by entry -----------------------------------------------------------
def exact(c, seed):
    s = prepare(c, seed)
    return {"window": _exact_attend, "tree": _exact_attend, "verify": _exact_verify, "pages": _exact_pages}[c["op"]](s, c)


def _exact_attend(s, c):
    lens, rows, pars = _lens(c), _rows(c), _parents(c) if c["op"] == "tree" else None
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    G, at = c["Hq"] // c["Hkv"], 0
    for i, (n, r) in enumerate(zip(lens, rows)):
        sees = torch.zeros(r, n + r, dtype=torch.bool, device="cuda")
        w = c["window"] or 1 << 40
        depth = _depths(pars[i]) if pars else list(range(r))
        pos = n + torch.tensor(depth, device="cuda")[:, None]
        j = torch.arange(n + r, device="cuda")[None]
        if pars:
            sees[:, :n] = ((j > pos - w) | (j < c["sinks"]))[:, :n]
            for t in range(r):
                a = t
                while a >= 0:
                    sees[t, n + a] = True
                    a = pars[i][a]
        else:
            sees = (j <= pos) & ((j > pos - w) | (j < c["sinks"]))
        pages = s["table"][i, :-(-(n + r) // c["page"])].long()
        for h in range(c["Hkv"]):
            k = s["k"][0, pages, h].reshape(-1, c["D"])[:n + r].double()
            v = s["v"][0, pages, h].reshape(-1, c["D"])[:n + r].double()
            for g in range(G):
                z = s["q"][at:at + r, h * G + g].double() @ k.t().contiguous() / math.sqrt(c["D"])
                z[~sees] = -math.inf
                out[at:at + r, h * G + g] = torch.softmax(z, -1) @ v
        at += r
    return out


def _exact_verify(s, c):
    rows, pars = _rows(c), _parents(c)
    token = s["tokens"].tolist()
    u, us = s["u"].tolist(), s["u_sample"].tolist()
    keep, path, drawn, at = [], [], [], 0
    for e, r in enumerate(rows):
        node, way = 0, [0]
        while True:
            p, q = s["p"][at + node].double(), s["q"][at + node].double()
            rest, mass, nxt = p, 1.0, None           # what is left of the target, not normalised, and its sum
            lam = 0.0
            for kid in [t for t in range(r) if pars[e][t] == node]:
                x = token[at + kid]
                if u[at + kid] * float(q[x]) * mass < float(rest[x]):
                    nxt = kid
                    break
                lam += mass
                rest = torch.relu(p - lam * q)
                mass = float(rest.sum())
            if nxt is None:
                break
            node = nxt
            way.append(node)
        if not float(rest.sum()) > 0:
            rest = p
        cum = torch.cumsum(rest, 0)
        over = torch.nonzero(cum > us[e] * cum[-1])
        drawn.append(int(over[0]) if len(over) else int(torch.nonzero(rest > 0)[-1]))
        keep.append(len(way))
        path += way + [-1] * (r - len(way))
        at += r
    return _ints(keep), _ints(path), _ints(drawn)


def _exact_pages(s, c):
    """The moves one after the other, on lists; None for caches that are too large to go through twice."""
    page, rows, keeps, small = c["page"], _rows(c), _keeps(c), s["k"].numel() < 1 << 28
    table, refs, size = s["table"].tolist(), s["refs"].tolist(), s["seq_len"].tolist()
    path, dst, src = s["path"].tolist(), s["dst"].tolist(), s["src"].tolist()
    for a, b in zip(src, dst):
        for i in range(-(-size[a] // page)):
            table[b][i] = table[a][i]
            refs[table[b][i]] += 1
        size[b] = size[a]
    free = [i for i, r in enumerate(refs) if r == 0]
    shared = [r > 1 for r in refs]
    granted, asked, at, got = [], 0, 0, []
    for b, r in zip(dst, rows):
        want = [i for i in range(size[b] // page, -(-(size[b] + r) // page)) if table[b][i] < 0 or shared[table[b][i]]]
        ok = not want or asked + len(want) <= len(free)
        granted.append(int(ok))
        for w, i in enumerate(want if ok else []):
            new, old = free[asked + w], table[b][i]
            if old >= 0:
                m = size[b] % page
                if small:
                    s["k"][:, new, :, :m] = s["k"][:, old, :, :m]
                    s["v"][:, new, :, :m] = s["v"][:, old, :, :m]
                refs[old] -= 1
            refs[new] += 1
            got.append((b, i, new))
            table[b][i] = new
        asked += len(want)
    for b, r, m in zip(dst, rows, keeps):
        n = size[b]
        for row in range(r if small else 0):
            pg, sl = table[b][(n + row) // page], (n + row) % page
            s["k"][:, pg, :, sl] = s["new_k"][:, at + row]
            s["v"][:, pg, :, sl] = s["new_v"][:, at + row]
        for to in range(m if small else 0):
            frm = at + path[at + to]
            pg, sl = table[b][(n + to) // page], (n + to) % page
            s["k"][:, pg, :, sl] = s["new_k"][:, frm]
            s["v"][:, pg, :, sl] = s["new_v"][:, frm]
        size[b] = n + m
        for i in range(-(-size[b] // page), len(table[b])):
            if table[b][i] >= 0:
                refs[table[b][i]] -= 1
                table[b][i] = -1
        at += r
    k, v = (s["k"].double(), s["v"].double()) if small else (None, None)
    return k, v, _ints(table), _ints(size), _ints(refs), _ints(granted)
