"""What is timed when the rest of a decode step is looked at, from the projections to the next token: rows turned to
their positions, alone and on their way into the paged cache, the choice of the blocks of a long context that a query
reads and the attention over them, the bounds that the choice goes by, and tokens drawn from logits.

A case is a dict of plain values:
  op      "rotate", "append", "sparse" (choice and attention), "bounds" or "sample"
  dtype   "bf16" or "f32": the cache, queries, rows and outputs (sample: the logits)
  B       batch entries, sequences (rotate, sample: rows);   T  most rows of an entry
  L       most tokens that an entry has in the cache before its rows (rotate: the farthest position)
  tree    the rows of an entry are nodes of a tree of drafts, not successive tokens
  Hq, Hkv, D   query heads, key/value heads, head dimension
  dims, layout, scaling   what of a head is turned, how its pairs lie, how the angles are scaled
  page    slots of a page;   slot_major  the cache stores [page][slot][head], else [page][head][slot]
  block, select, sinks, recent   positions of a block, blocks that a row chooses, positions that are always read
  layers, back   bounds: layers of the cache, committed positions of each sequence that are new
  V, cut, probs  sample: vocabulary, which cuts the rows ask for, what becomes of the probabilities ("", "bf16", "f32")
  ragged  entries differ in length and rows
Where `own` is false, run() computes the plain form; where it is true, it calls the package.
"""
import math

import torch

own = False

GOLD = 0.6180339887498949


def listed():
    return [
        # the draft's queries of one tree, interleaved pairs, full precision: a launch and little else
        dict(name="rotate f32 7 rows", op="rotate", dtype="f32", B=7, T=1, L=1500, Hq=32, D=96, dims=96, layout="interleaved",
             scaling="none", ragged=False),
        # a long prompt's rows, half of each head turned, contexts stretched part by part: copies of them
        dict(name="rotate bf16 8192 rows", op="rotate", dtype="bf16", B=8192, T=1, L=1000000, Hq=40, D=128, dims=64, layout="half",
             scaling="parts", ragged=False),
        # drafted trees of three short sequences, a quarter of each head turned
        dict(name="append tree f32 3x7", op="append", dtype="f32", B=3, T=7, L=1500, tree=True, Hq=32, Hkv=32, D=96, dims=24,
             layout="interleaved", scaling="none", page=32, slot_major=True, ragged=True),
        # two pieces of prompts, odd lengths
        dict(name="append prompt 2x4095", op="append", dtype="bf16", B=2, T=4095, L=4097, tree=False, Hq=40, Hkv=10, D=128, dims=128,
             layout="half", scaling="linear", page=32, slot_major=False, ragged=True),
        # the next token of two chats: latency
        dict(name="sparse 2 tokens over 3k", op="sparse", dtype="bf16", B=2, T=1, L=3001, tree=False, Hq=32, Hkv=8, D=128, page=16,
             slot_major=False, block=16, select=32, sinks=4, recent=64, ragged=True),
        # a serving batch of single tokens over long documents
        dict(name="sparse 16 tokens over 64k", op="sparse", dtype="bf16", B=16, T=1, L=65535, tree=False, Hq=40, Hkv=10, D=128, page=64,
             slot_major=False, block=32, select=64, sinks=4, recent=512, ragged=True),
        # drafted trees in full precision, every head its own cache
        dict(name="sparse trees f32 3x7 over 20k", op="sparse", dtype="f32", B=3, T=7, L=20011, tree=True, Hq=32, Hkv=32, D=96, page=32,
             slot_major=True, block=32, select=24, sinks=2, recent=100, ragged=True),
        # after a decode step: the pages that became full in six sequences, all layers
        dict(name="bounds after a step", op="bounds", dtype="bf16", B=6, L=1900, Hkv=8, D=128, page=16, slot_major=False, block=16,
             layers=32, back=8, ragged=True),
        # after a prompt: all pages of two long documents
        dict(name="bounds of 2x48k", op="bounds", dtype="bf16", B=2, L=49152, Hkv=10, D=128, page=64, slot_major=True, block=32,
             layers=2, back=49152, ragged=True),
        # one sequence's token, a small vocabulary, and the probabilities that a draft is verified against
        dict(name="sample 1 of 32064", op="sample", dtype="f32", B=1, V=32064, cut="k", probs="f32", ragged=False),
        # a serving batch, every user with their own settings
        dict(name="sample bf16 64 of 128256", op="sample", dtype="bf16", B=64, V=128256, cut="mix", probs="", ragged=False),
        # all nodes of a large batch of trees: the target's probabilities
        dict(name="sample 512 of 128256", op="sample", dtype="f32", B=512, V=128256, cut="p", probs="f32", ragged=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _most(op, key):
    return max(work(c)[key] for c in listed() if c["op"] == op)


def _turned(rng, c):
    c["layout"] = rng.choice(["half", "interleaved"])
    c["dims"] = rng.choice([c["D"], c["D"], c["D"] // 2, c["D"] // 4, 2 * rng.randint(1, c["D"] // 2)])
    c["scaling"] = rng.choice(["none", "linear", "base", "parts", "list"])


def draw(rng):
    op = rng.choice(["rotate", "append", "sparse", "sparse", "bounds", "sample", "sample"])
    while True:
        c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "f32"]), ragged=rng.random() < 0.7)
        if op == "sample":
            c.update(B=_log(rng, 1, 512), V=_log(rng, 1000, 128256), cut=rng.choice(["none", "k", "p", "min", "mix"]),
                     probs=rng.choice(["", "bf16", "f32"]))
        elif op == "rotate":
            c.update(B=_log(rng, 1, 8192), T=1, L=_log(rng, 10, 1000000), Hq=rng.choice([1, 3, 8, 32, 40]), D=rng.choice([64, 96, 128]))
            _turned(rng, c)
        else:
            c.update(page=rng.choice([16, 32, 64, 128]), slot_major=rng.random() < 0.4, D=rng.choice([64, 96, 128, 128]),
                     Hkv=rng.choice([1, 2, 4, 8, 8, 10, 16, 32]))
            c["block"] = rng.choice([b for b in (16, 32, 64, 128) if b <= c["page"]])
            if op == "bounds":
                c.update(B=_log(rng, 1, 16), L=_log(rng, 1, 49152), layers=_log(rng, 1, 32), back=_log(rng, 1, 49152))
            else:
                c["Hq"] = c["Hkv"] * rng.choice([1, 2, 3, 4, 5, 7, 8])
                c["tree"] = rng.random() < 0.4
                if op == "append":
                    c.update(B=_log(rng, 1, 32), T=_log(rng, 1, 64 if c["tree"] else 4095), L=_log(rng, 1, 4097))
                    _turned(rng, c)
                else:
                    c.update(B=_log(rng, 1, 16), T=_log(rng, 1, 16) if rng.random() < 0.5 else 1, L=_log(rng, 1, 65535),
                             select=_log(rng, 1, 128), sinks=rng.randint(0, 40), recent=_log(rng, 1, 1024))
        w = work(c)
        if w["bytes"] > _most(op, "bytes") or w["flops"] > _most(op, "flops"):
            continue
        if op == "sparse" and (c["D"] * (sum(_rows(c)) * c["Hkv"] * _most_read(c) + c["B"] * c["Hkv"] * c["L"] // 16) > 1 << 29 or
                               sum(_rows(c)) * c["Hq"] * c["L"] // c["block"] > 40 * 16 * 4096):
            continue                                  # (the plain form's gathered keys and scores)
        if "page" in c and c.get("layers", 1) * _n_pages(c) * c["page"] * c["Hkv"] * c["D"] > 1 << 31:
            continue
        return c


# ---- the entries of a case: fixed by the case alone, so that work() knows them --------------------
def _lens(c):
    """Tokens of each sequence in the cache; the first has L."""
    return [c["L"] if i == 0 or not c["ragged"] else max(1, int(c["L"] * (1 - 0.9 * ((i * GOLD) % 1.0)))) for i in range(c["B"])]


def _rows(c):
    """Rows of each entry; the first has T."""
    if c["op"] == "bounds":
        return [0] * c["B"]
    return [c["T"] if i == 0 or not c["ragged"] else max(1, int(c["T"] * (1 - 0.7 * ((i * GOLD * GOLD) % 1.0)))) for i in range(c["B"])]


def _need(c):
    """Pages that each entry holds, its rows included."""
    return [-(-(n + r) // c["page"]) for n, r in zip(_lens(c), _rows(c))]


def _n_pages(c):
    return sum(_need(c)) + 7


def _parents(c):
    """Parent of each node, per entry: node 0 is the last committed token, nobody has more than three children."""
    out = []
    for e, n in enumerate(_rows(c)):
        par, kids = [-1], [0]
        for t in range(1, n):
            at = int((((t + 3 * e) * GOLD) % 1.0) * t)
            while kids[at] >= 3:
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


def _parts(c, n):
    """(end of the sinks, start of the tail) of a sequence of n tokens, whole blocks."""
    tail = min(max(0, n - c["recent"]), n - n % c["page"]) // c["block"] * c["block"]
    return min(-(-c["sinks"] // c["block"]) * c["block"], tail), tail


def _most_read(c):
    """Most positions that a row reads."""
    most = 0
    for n, r in zip(_lens(c), _rows(c)):
        sinks, tail = _parts(c, n)
        most = max(most, sinks + min(c["select"] * c["block"], tail - sinks) + n - tail + r)
    return most


def work(c):
    es = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "sample":
        out = {"": 0, "bf16": 2, "f32": 4}[c["probs"]]
        return {"bytes": c["B"] * (c["V"] * (es + out) + 24), "flops": 6 * c["B"] * c["V"]}
    if c["op"] == "rotate":
        return {"bytes": c["B"] * (2 * c["Hq"] * c["D"] * es + 4) + 4 * c["dims"], "flops": 3 * c["B"] * c["Hq"] * c["dims"]}
    if c["op"] == "append":
        n = sum(_rows(c))
        return {"bytes": n * 2 * (c["Hq"] + 2 * c["Hkv"]) * c["D"] * es + 4 * c["dims"], "flops": 3 * n * (c["Hq"] + c["Hkv"]) * c["dims"]}
    if c["op"] == "bounds":
        pages = sum(n // c["page"] - max(0, n - c["back"]) // c["page"] for n in _lens(c))
        row = c["layers"] * c["Hkv"] * c["D"] * es
        return {"bytes": max(1, pages * row * (c["page"] + 2 * (c["page"] // c["block"]))), "flops": max(1, 2 * pages * row // es * c["page"])}
    by = fl = 0
    for n, r in zip(_lens(c), _rows(c)):
        sinks, tail = _parts(c, n)
        blocks = (tail - sinks) // c["block"]
        chosen = min(c["select"], blocks)
        always = sinks + n - tail + r
        by += c["Hkv"] * c["D"] * es * (2 * blocks + 2 * r * chosen * c["block"] + 2 * always) + r * (2 * c["Hq"] * c["D"] * es + 4 * c["Hkv"] * c["select"])
        fl += 4 * c["D"] * c["Hq"] * r * (blocks + chosen * c["block"] + always)
    return {"bytes": by, "flops": fl}


# ---- inputs ---------------------------------------------------------------------------------------
def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _starts(rows):
    s = [0]
    for r in rows:
        s.append(s[-1] + r)
    return _ints(s)


SCALED = dict(factor=8.0, slow=1.0, fast=32.0, original=4096.0)


def _angles(c):
    """Angles per position of each pair, in 64 bits: what a program works out once for its model."""
    i = torch.arange(c["dims"] // 2, dtype=torch.float64, device="cuda")
    base, f = 10000.0, SCALED["factor"]
    if c["scaling"] == "base" and c["dims"] > 2:
        base *= f ** (c["dims"] / (c["dims"] - 2))
    a = base ** (-2 * i / c["dims"])
    if c["scaling"] == "linear":
        a = a / f
    if c["scaling"] == "parts":                       # whole turns within the original length stay, less than one is stretched
        mix = ((SCALED["original"] * a / (2 * math.pi) - SCALED["slow"]) / (SCALED["fast"] - SCALED["slow"])).clamp(0, 1)
        a = a * mix + a / f * (1 - mix)
    if c["scaling"] == "list":
        a = a / (1 + 0.37 * i)
    return a


def _cache(c, g, s, keys):
    """A cache whose pages lie scattered, as after hours of serving."""
    lens, need, P, H, D = _lens(c), _need(c), _n_pages(c), c["Hkv"], c["D"]
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    order = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(need)), -1, dtype=torch.int32, device="cuda")
    used = 0
    for i, k in enumerate(need):
        table[i, :k] = order[used:used + k]
        used += k
    refs = torch.zeros(P, dtype=torch.int32, device="cuda")
    refs[order[:used].long()] = 1
    shape = (c.get("layers", 1), P, c["page"], H, D) if c["slot_major"] else (c.get("layers", 1), P, H, c["page"], D)
    k, v = (torch.empty(shape, dtype=dt, device="cuda").normal_(generator=g) for _ in range(2))
    if c["slot_major"]:
        k, v = k.transpose(2, 3), v.transpose(2, 3)
    if keys:                                          # a few loud channels, and what a page is about
        wide = torch.exp(0.4 * torch.randn(D, generator=g, device="cuda"))
        about = 0.5 * torch.randn(shape[0], P, H, 1, D, generator=g, device="cuda")
        k.mul_(wide.to(dt)).add_(about.to(dt))
    s.update(k=k, v=v, table=table, refs=refs, seq_len=_ints(lens), seqs=torch.arange(len(lens), dtype=torch.int32, device="cuda"),
             max_len=max(n + r for n, r in zip(lens, _rows(c))))


def _bounds_of(c, k):
    """[layers][pages][heads][blocks of a page][lo, hi][D] of all pages."""
    x = k.unflatten(3, (c["page"] // c["block"], c["block"]))
    return torch.stack([x.amin(4), x.amax(4)], 4).contiguous()


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    uniform = lambda *shape: torch.rand(shape, generator=g, device="cuda")
    s = {"case": c}
    if c["op"] == "sample":
        B, V, cut = c["B"], c["V"], c["cut"]
        x = 2.5 * normal(B, V)
        x += 5.0 * (uniform(B, V) < 8.0 / V)          # a few words that fit, and some that are forbidden
        x[uniform(B, V) < 0.01] = -math.inf
        s["logits"] = x.to(dt)
        s["u"] = uniform(B)
        pick = lambda wanted, some, off: torch.where(uniform(B) < wanted, some, torch.full_like(some, off))
        share = {"mix": 0.6}.get(cut, 1.0)
        s["temperature"] = pick(0.9 if cut == "mix" else 1.0, 0.5 + 0.8 * uniform(B), 0.0)
        s["top_k"] = pick(share, torch.exp(1 + 6 * uniform(B)).to(torch.int32), 0) if cut in ("k", "mix") else None
        s["top_p"] = pick(share, 0.8 + 0.19 * uniform(B), 1.0) if cut in ("p", "mix") else None
        s["min_p"] = pick(share, 0.02 + 0.1 * uniform(B), 0.0) if cut in ("min", "mix") else None
        return s
    if c["op"] == "rotate":
        s["x"] = normal(c["B"], c["Hq"], c["D"]).to(dt)
        s["positions"] = torch.randint(0, c["L"] + 1, (c["B"],), generator=g, device="cuda").to(torch.int32)
        s["angles"] = _angles(c)
        return s
    _cache(c, g, s, keys=c["op"] == "sparse")
    if c["op"] == "bounds":
        s["bounds"] = torch.zeros(c["layers"], _n_pages(c), c["Hkv"], c["page"] // c["block"], 2, c["D"], dtype=dt, device="cuda")
        return s
    rows = _rows(c)
    n = sum(rows)
    s.update(row_start=_starts(rows), n_rows=n, max_rows=max(rows))
    s["parents"] = _ints([p for par in _parents(c) for p in par]) if c["tree"] else None
    if c["op"] == "append":
        fused = normal(n, c["Hq"] + 2 * c["Hkv"], c["D"]).to(dt)       # one projection's output, queries, keys and values side by side
        s["q"], s["new_k"], s["new_v"] = fused.split([c["Hq"], c["Hkv"], c["Hkv"]], 1)
        s["angles"] = _angles(c)
    else:
        s["q"] = (1.5 * normal(n, c["Hq"], c["D"])).to(dt)
        s["bounds"] = _bounds_of(c, s["k"])
    return s


# ---- the package's calls ----------------------------------------------------------------------------
def _handles(s):
    """What a program keeps beside its data: descriptors, output buffers, workspace."""
    import paper_2412_01380_amd as A
    c = s["case"]
    h = {"A": A}
    ints = lambda *m: torch.empty(m, dtype=torch.int32, device="cuda")
    size = 0
    if c["op"] == "sample":
        h["token"] = ints(c["B"])
        if c["probs"]:
            h["probs"] = torch.empty(c["B"], c["V"], dtype=torch.bfloat16 if c["probs"] == "bf16" else torch.float32, device="cuda")
        size = A.dip_sample_workspace_bytes(c["B"], c["V"])
    if c["op"] in ("rotate", "append"):
        h["rot"] = A.Rotary(s["angles"], A.DIP_ROTARY_HALF if c["layout"] == "half" else A.DIP_ROTARY_INTERLEAVED)
        h["out"] = torch.empty(s["x"].shape if c["op"] == "rotate" else s["q"].shape, dtype=s["x" if c["op"] == "rotate" else "q"].dtype, device="cuda")
    if c["op"] in ("append", "sparse", "bounds"):
        h["cache"] = A.KvCache(s["k"], s["v"], s["table"], s["seq_len"], s["refs"])
    if c["op"] in ("append", "sparse"):
        h["batch"] = A.Batch(s["row_start"], s["n_rows"], s["max_rows"], seqs=s["seqs"], max_len=s["max_len"])
    if c["op"] == "sparse":
        h["out"] = torch.empty_like(s["q"])
        h["blocks"] = ints(s["n_rows"], c["Hkv"], c["select"])
        size = max(A.dip_select_blocks_workspace_bytes(h["cache"], h["batch"], c["Hq"], c["block"]),
                   A.dip_block_attention_workspace_bytes(h["cache"], h["batch"], c["Hq"], c["block"], c["select"], c["sinks"], c["recent"]))
    h["ws"] = torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")
    return h


def _call(s):
    if "handles" not in s:
        s["handles"] = _handles(s)
    c, h = s["case"], s["handles"]
    A = h["A"]
    if c["op"] == "sample":
        A.dip_sample(s["logits"], s["u"], h["token"], h.get("probs"), h["ws"], temperature=s["temperature"], top_k=s["top_k"],
                     top_p=s["top_p"], min_p=s["min_p"])
        return (h["token"], h["probs"]) if c["probs"] else h["token"]
    if c["op"] == "rotate":
        A.dip_rotate_rows(h["rot"], s["x"], s["positions"], h["out"])
        return h["out"]
    if c["op"] == "append":
        A.dip_kv_append_rotary(h["cache"], 0, h["batch"], s["parents"], h["rot"], s["q"], h["out"], s["new_k"], s["new_v"])
        return s["k"], s["v"], h["out"]
    if c["op"] == "bounds":
        A.dip_kv_block_bounds(h["cache"], 0, c["layers"], s["seqs"], c["back"], s["bounds"])
        return s["bounds"]
    A.dip_select_blocks(h["cache"], 0, h["batch"], s["q"], s["bounds"], c["sinks"], c["recent"], h["blocks"], h["ws"])
    A.dip_block_attention(h["cache"], 0, h["batch"], s["parents"], h["blocks"], c["block"], s["q"], 1 / math.sqrt(c["D"]), c["sinks"],
                          c["recent"], h["out"], h["ws"])
    return h["blocks"], h["out"]


def run(s):
    if own:
        return _call(s)
    return {"rotate": _rotate, "append": _append, "bounds": _bounds, "sparse": _sparse, "sample": _sample}[s["case"]["op"]](s)


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


def _turn(x, positions, angles, layout):
    """Angles in 64 bits (a position of a million turns leaves few bits of an fp32 one), the rest in 32."""
    a = positions.double()[:, None, None] * angles
    co, si = a.cos().float(), a.sin().float()
    y = x.float()
    d = 2 * angles.shape[0]
    y, rest = y[..., :d], y[..., d:]
    if layout == "half":
        p, q = y[..., :d // 2], y[..., d // 2:]
        y = torch.cat([p * co - q * si, p * si + q * co, rest], -1)
    else:
        p, q = y[..., 0::2], y[..., 1::2]
        y = torch.cat([torch.stack([p * co - q * si, p * si + q * co], -1).flatten(-2), rest], -1)
    return y.to(x.dtype)


def _rotate(s):
    return _turn(s["x"], s["positions"], s["angles"], s["case"]["layout"])


def _append(s):
    c = s["case"]
    b, t = _of_rows(s)
    n = s["seq_len"].long()[b]
    place = n + t
    pos = place
    if c["tree"]:
        pos = n + (_ancestors(s["parents"], b, t, c["B"], s["max_rows"]).sum(-1) - 1)[b, t]
    page, slot = s["table"][b, place // c["page"]].long(), place % c["page"]
    s["k"][0, page, :, slot] = _turn(s["new_k"], pos, s["angles"], c["layout"])
    s["v"][0, page, :, slot] = s["new_v"]
    return s["k"], s["v"], _turn(s["q"], pos, s["angles"], c["layout"])


def _bounds(s):
    c = s["case"]
    n, j = s["seq_len"].long()[:, None], torch.arange(s["table"].shape[1], device="cuda")[None]
    mine = (j < n // c["page"]) & ((j + 1) * c["page"] > n - c["back"])
    at = s["table"][mine].long()
    if at.numel():
        s["bounds"][:, at] = _bounds_of(c, s["k"][:, at])
    return s["bounds"]


def _sparse(s):
    c = s["case"]
    B, T, Hq, H, D, blk, sel = c["B"], s["max_rows"], c["Hq"], c["Hkv"], c["D"], c["block"], c["select"]
    G = Hq // H
    b, t = _of_rows(s)
    n = s["seq_len"].long()
    tail = torch.minimum((n - c["recent"]).clamp(min=0), n - n % c["page"]) // blk * blk
    sink = torch.minimum(torch.full_like(tail, -(-c["sinks"] // blk) * blk), tail)
    # scores of all blocks, in 64 bits: which ones are chosen must not hang on the order of a sum
    pages = s["table"].clamp(min=0).long()
    bound = s["bounds"][0][pages].transpose(1, 2).reshape(B, H, -1, 2, D)      # [B, H, blocks, 2, D]
    q = torch.zeros(B, T, Hq, D, device="cuda", dtype=torch.float64)
    q[b, t] = s["q"].double()
    q = q.view(B, T, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, T * G, D)
    score = torch.matmul(q.clamp(min=0), bound[..., 1, :].double().transpose(2, 3).contiguous())
    score -= torch.matmul((-q).clamp(min=0), bound[..., 0, :].double().transpose(2, 3).contiguous())
    score = score.view(B, H, T, G, -1).amax(3).float()
    score = score.permute(0, 2, 1, 3)[b, t]                                     # [rows, H, blocks]
    j = torch.arange(score.shape[-1], device="cuda")
    middle = ((j >= (sink // blk)[:, None]) & (j < (tail // blk)[:, None]))[b][:, None]
    order = torch.sort(score.masked_fill(~middle, -math.inf), dim=-1, descending=True, stable=True).indices[..., :sel]
    there = torch.arange(order.shape[-1], device="cuda") < middle.sum(-1, keepdim=True)
    far = score.shape[-1]
    order = torch.where(there, order, far).sort(-1).values
    chosen = torch.full((s["n_rows"], H, sel), -1, dtype=torch.int32, device="cuda")
    chosen[..., :order.shape[-1]] = torch.where(order < far, order, -1).int()
    # positions that a row reads: the sinks, the blocks, the tail and the step's own rows
    span = torch.arange(blk, device="cuda")
    blocks = (chosen.long()[..., None] * blk + span).flatten(-2)
    ok = (chosen >= 0)[..., None].expand(-1, -1, -1, blk).flatten(-2)
    front = torch.arange(-(-c["sinks"] // blk) * blk, device="cuda")
    back = torch.arange(int(c["recent"] + c["page"] + blk + T), device="cuda")
    at_back = tail[b, None] + back
    own_row = at_back - n[b, None]
    if c["tree"]:
        anc = _ancestors(s["parents"], b, t, B, T)[b, t]
        ok_back = (own_row < 0) | (torch.gather(anc, 1, own_row.clamp(0, T - 1)) & (own_row < T))
    else:
        ok_back = own_row <= t[:, None]
    R = s["n_rows"]
    wide = lambda x: x[:, None].expand(-1, H, -1)
    pos = torch.cat([wide(front.expand(R, -1)), blocks, wide(at_back)], -1)
    ok = torch.cat([wide(front[None] < sink[b, None]), ok, wide(ok_back)], -1)
    pos = torch.where(ok, pos, 0)
    page = torch.gather(s["table"][b].clamp(min=0).long()[:, None].expand(-1, H, -1), 2, pos // c["page"])
    head = torch.arange(H, device="cuda")[None, :, None]
    k = s["k"][0][page, head, pos % c["page"]].float()
    v = s["v"][0][page, head, pos % c["page"]].float()
    z = torch.matmul(s["q"].float().view(R, H, G, D), k.transpose(2, 3).contiguous()) / math.sqrt(D)
    z = z.masked_fill_(~ok[:, :, None], -math.inf)
    z = torch.exp(z - z.amax(-1, keepdim=True))
    z = z / z.sum(-1, keepdim=True)
    return chosen, torch.matmul(z, v).view(R, Hq, D).to(s["q"].dtype)


def _sample(s):
    """In 64 bits: a draw, or a cut, next to a border should not hang on rounding."""
    c = s["case"]
    x = s["logits"].double()
    temp = s["temperature"].double()[:, None]
    greedy = temp <= 0
    x, order = torch.sort(x, dim=1, descending=True, stable=True)
    w = torch.exp((x - x[:, :1]) / torch.where(greedy, torch.ones_like(temp), temp))
    rank = torch.arange(c["V"], device="cuda")[None]
    if s["top_k"] is not None:
        k = s["top_k"][:, None]
        w = torch.where((rank < k) | (k <= 0), w, 0.0)
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        up = torch.cumsum(w, 1)
        w = torch.where((up - w < p * up[:, -1:]) | (p >= 1), w, 0.0)
    if s["min_p"] is not None:
        w = torch.where(w >= s["min_p"].double()[:, None], w, 0.0)
    w = torch.zeros_like(w).scatter_(1, order, w)
    w = torch.where(greedy, torch.zeros_like(w).scatter_(1, order[:, :1], 1.0), w)
    up = torch.cumsum(w, 1)
    above = (up > s["u"].double()[:, None] * up[:, -1:]) & (w > 0)
    token = torch.where(above.any(1), above.int().argmax(1), (w > 0).int().cumsum(1).argmax(1)).to(torch.int32)
    if not c["probs"]:
        return token
    return token, (w / up[:, -1:]).to(torch.bfloat16 if c["probs"] == "bf16" else torch.float32)


# ---- the definitions in 64 bits, entry by entry -----------------------------------------------------------
def exact(c, seed):
    s = prepare(c, seed)
    return {"rotate": _exact_rotate, "append": _exact_append, "bounds": _exact_bounds, "sparse": _exact_sparse,
            "sample": _exact_sample}[c["op"]](s, c)


def _exact_turn(x, positions, angles, layout):
    """A pair as a complex number, times exp(i angle)."""
    out = x.double().clone()
    half = angles.shape[0]
    first = torch.arange(half, device="cuda") * (1 if layout == "half" else 2)
    second = first + (half if layout == "half" else 1)
    z = torch.complex(out[..., first], out[..., second])
    z = z * torch.polar(torch.ones(1, dtype=torch.float64, device="cuda"), positions.double()[:, None] * angles)[:, None]
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _exact_rotate(s, c):
    return _exact_turn(s["x"], s["positions"], s["angles"], c["layout"])


def _exact_append(s, c):
    k, v = s["k"].double(), s["v"].double()
    q, at = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), 0
    pars = _parents(c) if c["tree"] else None
    for i, (n, r) in enumerate(zip(_lens(c), _rows(c))):
        place = n + torch.arange(r, device="cuda")
        pos = n + torch.tensor(_depths(pars[i]), device="cuda") if pars else place
        page, slot = s["table"][i][place // c["page"]].long(), place % c["page"]
        k[0, page, :, slot] = _exact_turn(s["new_k"][at:at + r], pos, s["angles"], c["layout"])
        v[0, page, :, slot] = s["new_v"][at:at + r].double()
        q[at:at + r] = _exact_turn(s["q"][at:at + r], pos, s["angles"], c["layout"])
        at += r
    return k, v, q


def _exact_bounds(s, c):
    out = s["bounds"].double()
    for i, n in enumerate(_lens(c)):
        for j in range(max(0, n - c["back"]) // c["page"], n // c["page"]):
            page = int(s["table"][i, j])
            x = s["k"][:, page].unflatten(2, (c["page"] // c["block"], c["block"]))
            out[:, page, :, :, 0], out[:, page, :, :, 1] = x.amin(3).double(), x.amax(3).double()
    return out


def _exact_sparse(s, c):
    lens, rows, pars = _lens(c), _rows(c), _parents(c) if c["tree"] else None
    G, blk, at = c["Hq"] // c["Hkv"], c["block"], 0
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    chosen = torch.full((s["n_rows"], c["Hkv"], c["select"]), -1, dtype=torch.int32, device="cuda")
    for i, (n, r) in enumerate(zip(lens, rows)):
        sink, tail = _parts(c, n)
        pages = s["table"][i, :-(-(n + r) // c["page"])].long()
        own_rows = torch.zeros(r, r, dtype=torch.bool)
        for t in range(r):
            a = t
            while a >= 0:
                own_rows[t, a] = True
                a = pars[i][a] if pars else a - 1
        own_rows = own_rows.cuda()
        for h in range(c["Hkv"]):
            k = s["k"][0, pages, h].reshape(-1, c["D"])[:n + r].double()
            v = s["v"][0, pages, h].reshape(-1, c["D"])[:n + r].double()
            q = s["q"][at:at + r, h * G:(h + 1) * G].double()
            sees = torch.zeros(r, n + r, dtype=torch.bool, device="cuda")
            sees[:, :sink] = True
            sees[:, tail:n] = True
            sees[:, n:] = own_rows
            if tail > sink:
                b = s["bounds"][0, pages, h].reshape(-1, 2, c["D"])[sink // blk:tail // blk].double()
                score = torch.stack([torch.stack([torch.maximum(x * b[:, 0], x * b[:, 1]).sum(1) for x in y]).amax(0) for y in q]).float()
                take = min(c["select"], score.shape[1])
                best = torch.sort(-score, dim=1, stable=True).indices[:, :take].sort(1).values + sink // blk
                chosen[at:at + r, h, :take] = best.int()
                where = (best[:, :, None] * blk + torch.arange(blk, device="cuda")).view(r, -1)
                sees.scatter_(1, where, True)
            for g in range(G):
                z = (q[:, g] @ k.t().contiguous() / math.sqrt(c["D"])).masked_fill(~sees, -math.inf)
                out[at:at + r, h * G + g] = torch.softmax(z, -1) @ v
        at += r
    return chosen, out


def _exact_sample(s, c):
    """Row by row: the words in order of their logits, cut one rule after the other."""
    tokens, probs = [], torch.zeros(c["B"], c["V"], dtype=torch.float64, device="cuda") if c["probs"] else None
    get = lambda name, i, off: off if s[name] is None else s[name][i].item()
    for i in range(c["B"]):
        x = s["logits"][i].double()
        temp, k, p, m = s["temperature"][i].item(), get("top_k", i, 0), get("top_p", i, 1.0), get("min_p", i, 0.0)
        order = torch.sort(-x, stable=True).indices
        if temp <= 0:
            kept, w = order[:1], torch.ones(1, dtype=torch.float64, device="cuda")
        else:
            kept = order[:k] if k > 0 else order
            w = torch.exp((x[kept] - x[order[0]]) / temp)
            if p < 1:
                sums = torch.cumsum(w, 0)
                n = int((sums < p * sums[-1]).sum()) + 1
                kept, w = kept[:n], w[:n]
            kept, w = kept[w >= m], w[w >= m]
        full = torch.zeros(c["V"], dtype=torch.float64, device="cuda")
        full[kept] = w
        sums = torch.cumsum(full, 0)
        over = torch.nonzero(sums > s["u"][i].item() * sums[-1])
        tokens.append(int(over[0]) if len(over) else int(torch.nonzero(full)[-1]))
        if probs is not None:
            probs[i] = full / sums[-1]
    return (_ints(tokens), probs) if c["probs"] else _ints(tokens)
