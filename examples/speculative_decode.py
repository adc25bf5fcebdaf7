#!/usr/bin/env python3
"""Speculative decoding with pruned layers, end to end: a small random-weight decoder whose MLPs run as
DIP batches, whose attention reads a paged cache with a sliding window and sinks, or blocks of it that every row
chooses for itself, and whose drafts are trees that are verified against its own probabilities.

    python examples/speculative_decode.py [--tokens N] [--greedy] [--branches 2] [--blocks 8]

One step of the loop, for all sequences together:
    draft     a tree per sequence, at most 8 nodes of both together -- what dip_swiglu_mlp_forward_batched takes
    reserve   room for the nodes in the cache                     dip_kv_reserve
    layers    append keys and values, turned to their positions,  dip_kv_append_rotary,
              attend, MLP                                         dip_tree_attention (or dip_select_blocks and
                                                                  dip_block_attention), dip_swiglu_mlp_forward_batched
    verify    the probabilities, which nodes stand, next token    dip_sample, dip_verify_tree
    compact   keep their rows, give back the rest                 dip_kv_compact (and dip_kv_block_bounds)
The projections are torch products: the library has none.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2412_01380_amd as D  # noqa: E402

ROWS = 8          # rows that a batched MLP call takes


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def workspace(n):
    return torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")


class Decoder:
    """Pre-norm decoder layers in fp32 with a bf16 or fp32 cache; d_model is heads * head_dim."""

    def __init__(self, layers=2, heads=8, kv_heads=2, head_dim=64, d_ff=1536, vocab=512, keep=0.5, window=64, sinks=4,
                 dtype=torch.bfloat16, n_seqs=2, max_tokens=512, page=16, seed=0, blocks=0, recent=32):
        g = torch.Generator(device="cuda").manual_seed(seed)
        d = heads * head_dim
        normal = lambda *s, scale=1.0: torch.randn(s, generator=g, device="cuda") * scale
        self.heads, self.kv_heads, self.dim, self.d, self.vocab = heads, kv_heads, head_dim, d, vocab
        self.window, self.sinks, self.dtype = window, sinks, dtype
        self.blocks, self.recent, self.page = blocks, recent, page     # blocks: pages that a row chooses (0: the window)
        self.k_in, self.k_mid = max(1, int(keep * d)), max(1, int(keep * d_ff))
        self.emb = normal(vocab, d)
        # what a token leads to on its own: a fixed successor, more or less
        self.unemb = self.emb[torch.randperm(vocab, generator=g, device="cuda")] + normal(vocab, d, scale=0.5)
        self.qkv = [normal(d, (heads + 2 * kv_heads) * head_dim, scale=d ** -0.5) for _ in range(layers)]
        self.proj = [normal(d, d, scale=2.0 * d ** -0.5) for _ in range(layers)]
        self.mlps = [D.Mlp(D.Weight(normal(d, 2 * d_ff, scale=d ** -0.5).bfloat16()),
                           D.Weight(normal(d_ff, d, scale=2.0 * d_ff ** -0.5).bfloat16())) for _ in range(layers)]
        pages = n_seqs * max_tokens // page
        kv = lambda: torch.empty(layers, pages, kv_heads, page, head_dim, dtype=dtype, device="cuda")
        self.cache = D.KvCache(kv(), kv(), ints([[0] * (max_tokens // page)] * n_seqs), ints([0] * n_seqs), ints([0] * pages))
        D.dip_kv_init(self.cache)
        self.rot = D.Rotary(D.dip_rotary_frequencies(head_dim).cuda(), D.DIP_ROTARY_HALF)
        self.bounds = torch.zeros(layers, pages, kv_heads, 1, 2, head_dim, dtype=dtype, device="cuda")
        self.seqs, self.lens = ints(list(range(n_seqs))), [0] * n_seqs
        self.mlp_ws = workspace(max(D.dip_swiglu_mlp_forward_batched_workspace_bytes(self.mlps[0], b, self.k_in, self.k_mid)
                                    for b in range(1, ROWS + 1)))

    def batch(self, rows):
        starts = [0]
        for r in rows:
            starts.append(starts[-1] + r)
        return D.Batch(ints(starts), starts[-1], max(rows), seqs=self.seqs, max_len=max(n + r for n, r in zip(self.lens, rows)))

    def reserve(self, batch):
        granted = ints([0] * batch.n_batch)
        D.dip_kv_reserve(self.cache, batch, granted, workspace(D.dip_kv_reserve_workspace_bytes(self.cache, batch)))
        if not all(granted.tolist()):
            raise RuntimeError("the cache is full")

    def forward(self, batch, tokens, parents=None):
        """Logits behind each row; the rows' keys and values stay in the cache, not committed."""
        n, hd = batch.n_rows, self.heads * self.dim
        x = self.emb[tokens.long()]
        norm = lambda y: torch.nn.functional.rms_norm(y, (self.d,))
        if self.blocks:
            ws = workspace(max(D.dip_select_blocks_workspace_bytes(self.cache, batch, self.heads, self.page),
                               D.dip_block_attention_workspace_bytes(self.cache, batch, self.heads, self.page, self.blocks, self.sinks,
                                                                     self.recent)))
            chosen = torch.empty(n, self.kv_heads, self.blocks, dtype=torch.int32, device="cuda")
        else:
            ws = workspace(D.dip_attention_workspace_bytes(self.cache, batch, self.heads, self.window, self.sinks))
        for layer, (w_qkv, w_o, mlp) in enumerate(zip(self.qkv, self.proj, self.mlps)):
            fused = (norm(x) @ w_qkv).to(self.dtype)         # q, k and v side by side: the calls take strided rows
            k, v = fused[:, hd:].unflatten(1, (2, self.kv_heads, self.dim)).unbind(1)
            q, a = (torch.empty(n, self.heads, self.dim, dtype=self.dtype, device="cuda") for _ in range(2))
            D.dip_kv_append_rotary(self.cache, layer, batch, parents, self.rot, fused[:, :hd].unflatten(1, (self.heads, self.dim)), q, k, v)
            if self.blocks:
                D.dip_select_blocks(self.cache, layer, batch, q, self.bounds, self.sinks, self.recent, chosen, ws)
                D.dip_block_attention(self.cache, layer, batch, parents, chosen, self.page, q, self.dim ** -0.5, self.sinks, self.recent, a, ws)
            elif parents is None:
                D.dip_window_attention(self.cache, layer, batch, q, self.dim ** -0.5, self.window, self.sinks, a, ws)
            else:
                D.dip_tree_attention(self.cache, layer, batch, parents, q, self.dim ** -0.5, self.window, self.sinks, a, ws)
            x = x + a.view(n, hd).float() @ w_o
            h, y = norm(x), torch.empty_like(x)
            for r in range(0, n, ROWS):                       # (a prompt goes through in batches)
                b = min(ROWS, n - r)
                D.dip_swiglu_mlp_forward_batched(mlp, h[r:r + b], b, self.k_in, self.k_mid, None, None, 1.0, y[r:r + b], None,
                                                 None, None, self.mlp_ws)
            x = x + y
        return norm(x) @ self.unemb.t() * (9.0 / self.d)

    def commit(self, batch, path=None, keep=None):
        """Keep rows of a step, and work out the bounds of the pages that they filled."""
        D.dip_kv_compact(self.cache, batch, path, keep)
        if self.blocks:
            D.dip_kv_block_bounds(self.cache, 0, len(self.mlps), self.seqs, batch.c.max_rows, self.bounds)

    def draft_logits(self, token):
        """The drafter: the model without its layers."""
        return torch.nn.functional.rms_norm(self.emb[token], (self.d,)) @ self.unemb.t() * (9.0 / self.d)


def probabilities(logits, greedy, top_p=0.95):
    """What tokens are drawn from, for the target and the drafter alike."""
    rows = logits.view(-1, logits.shape[-1])
    probs = torch.empty_like(rows)
    each = lambda x: torch.full((len(rows),), x, device="cuda")
    D.dip_sample(rows, None, None, probs, workspace(D.dip_sample_workspace_bytes(*rows.shape)), temperature=each(0.0 if greedy else 1.0),
                 top_p=each(top_p))
    return probs.view_as(logits)


def generate(model, prompts, n_tokens, nodes=4, branches=1, greedy=False, seed=0):
    """n_tokens new tokens (or a few more) for each prompt.  nodes: of a sequence's tree, its root -- the last
    token -- among them; branches: drafts of one node.  Returns (tokens per sequence, model steps)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    uniform = lambda n: torch.rand(n, generator=g, device="cuda")
    B = len(prompts)
    assert 1 <= nodes and B * nodes <= ROWS
    # the prompts but for their last tokens, in one go
    rows = [len(p) - 1 for p in prompts]
    batch = model.batch(rows)
    model.reserve(batch)
    model.forward(batch, ints([t for p in prompts for t in p[:-1]]))
    model.commit(batch)
    model.lens = [n + r for n, r in zip(model.lens, rows)]
    out, steps = [list(p) for p in prompts], 0
    parents = [-1] + [(t - 1) // branches for t in range(1, nodes)]
    while min(len(o) - len(p) for o, p in zip(out, prompts)) < n_tokens:
        # a tree per sequence: breadth first, every node's children drawn from the drafter behind it
        tokens, q = [], []
        for o in out:
            tree = [o[-1]]
            rows_q = []
            for t in range(nodes):
                rows_q.append(probabilities(model.draft_logits(tree[t]), greedy))
                kids = sum(p == t for p in parents)
                tree += torch.multinomial(rows_q[-1], kids, replacement=True, generator=g).tolist() if kids else []
            tokens += tree
            q += rows_q
        batch = model.batch([nodes] * B)
        model.reserve(batch)
        tok, par = ints(tokens), ints(parents * B)
        p = probabilities(model.forward(batch, tok, par), greedy)
        keep, path, token = ints([0] * B), ints([0] * B * nodes), ints([0] * B)
        kids = max(1, branches)
        ws = workspace(D.dip_verify_tree_workspace_bytes(batch, model.vocab, kids))
        D.dip_verify_tree(batch, tok, par, p, torch.stack(q), uniform(B * nodes), uniform(B), kids, keep, path, token, ws)
        model.commit(batch, path, keep)
        steps += 1
        for i, (n, x) in enumerate(zip(keep.tolist(), token.tolist())):
            out[i] += [tokens[i * nodes + t] for t in path[i * nodes + 1:i * nodes + n].tolist()] + [x]
            model.lens[i] += n
    return out, steps


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--nodes", type=int, default=4)
    ap.add_argument("--branches", type=int, default=1)
    ap.add_argument("--greedy", action="store_true")
    ap.add_argument("--blocks", type=int, default=0, help="pages that a row chooses, in place of the window")
    a = ap.parse_args()
    prompts = [[1, 2, 3, 4, 5, 6, 7], [100, 90, 80]]
    one, one_steps = generate(Decoder(blocks=a.blocks), prompts, a.tokens, nodes=1, greedy=a.greedy)
    out, steps = generate(Decoder(blocks=a.blocks), prompts, a.tokens, a.nodes, a.branches, a.greedy)
    made = sum(len(o) for o in out) - sum(len(p) for p in prompts)
    print(f"{made} tokens in {steps} steps of {len(prompts)} x {a.nodes} rows: {made / steps / len(prompts):.2f} tokens a step "
          f"and sequence (one token at a time: {one_steps} steps)")
    if a.greedy:
        same = all(x[:len(p) + a.tokens] == y[:len(p) + a.tokens] for x, y, p in zip(out, one, prompts))
        print("the same tokens as one at a time:", same)


if __name__ == "__main__":
    main()
