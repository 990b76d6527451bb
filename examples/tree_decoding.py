"""Draft-tree decoding of a small decoder over the paged 4-bit cache.

The loop of Algorithm 1 with the target model run by this package's own cache: a prompt is
stored and its alignment table sampled; then, step by step, candidates are drafted and merged
into a tree (Eq. 2), the tree's nodes run through the model in one pass (``kv_plan`` once,
``kv_write`` and ``kv_attend`` per layer), the tree is verified and the accepted path's entries
are moved into place (``kv_commit``).  The weights are random: what the tokens say means nothing,
but strict verification emits exactly the tokens of decoding one by one, which is what is compared.

    python examples/tree_decoding.py
"""
from __future__ import annotations

import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2505_13204_b200 import binding                                     # noqa: E402

PAGE = binding.KV_PAGE


class Model:
    """Pre-norm decoder with grouped heads, head norms and rotary positions; fp32."""

    def __init__(self, ctx, layers=2, hidden=256, q_heads=8, kv_heads=2, head_dim=64, vocab=512, max_positions=1024, seed=0):
        g = torch.Generator().manual_seed(seed)

        def rand(*shape, scale=1.0):
            return (torch.randn(shape, generator=g) * scale).to(ctx.device)

        self.ctx, self.layers, self.head_dim, self.q_heads, self.kv_heads, self.vocab = ctx, layers, head_dim, q_heads, kv_heads, vocab
        self.embed, self.unembed = rand(vocab, hidden), rand(hidden, vocab, scale=hidden ** -0.5)
        self.wqkv = [rand(hidden, (q_heads + 2 * kv_heads) * head_dim, scale=hidden ** -0.5) for _ in range(layers)]
        self.wo = [rand(q_heads * head_dim, hidden, scale=(q_heads * head_dim) ** -0.5) for _ in range(layers)]
        self.w1 = [rand(hidden, 2 * hidden, scale=hidden ** -0.5) for _ in range(layers)]
        self.w2 = [rand(2 * hidden, hidden, scale=(2 * hidden) ** -0.5) for _ in range(layers)]
        self.qn = [1 + rand(head_dim, scale=0.1) for _ in range(layers)]
        self.kn = [1 + rand(head_dim, scale=0.1) for _ in range(layers)]
        angle = torch.arange(max_positions)[:, None] * 10000.0 ** (-torch.arange(0, head_dim, 2) / head_dim)
        self.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float().contiguous().to(ctx.device)

    @staticmethod
    def norm(x):
        return x * torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + 1e-6)

    def __call__(self, cache, tokens, plan, rows_per_seq=0, node_parent=None):
        """Logits of the token rows that ``plan`` has placed; rows of NONE are padding."""
        ctx, D, Hq, Hk = self.ctx, self.head_dim, self.q_heads, self.kv_heads
        x = self.embed[tokens.clamp(min=0).long()]
        for l in range(self.layers):
            qkv = (self.norm(x) @ self.wqkv[l]).view(-1, Hq + 2 * Hk, D)
            q = ctx.kv_write(cache.pages[l], qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:], plan["slot_map"], plan["positions"],
                             self.cos_sin, self.qn[l], self.kn[l])["q"]
            o = ctx.kv_attend(q, cache.pages[l], cache.table, cache.length, plan["kv_len"],
                              None if rows_per_seq else plan["tok_offsets"], rows_per_seq, node_parent)["out"]
            x = x + o.flatten(1) @ self.wo[l]
            x = x + torch.nn.functional.gelu(self.norm(x) @ self.w1[l]) @ self.w2[l]
        return self.norm(x) @ self.unembed


class Cache:
    """Page pools of all layers, the page tables and what each sequence has in them."""

    def __init__(self, model, n_seqs, n_pages, max_pages):
        dev = model.ctx.device
        self.ctx = model.ctx
        self.pages = binding.kv_pages(n_pages, model.kv_heads, model.head_dim, layers=model.layers, device=dev)
        self.table = torch.full((n_seqs, max_pages), binding.NONE, dtype=torch.int32, device=dev)
        self.held = torch.zeros(n_seqs, dtype=torch.int32, device=dev)
        self.free = torch.arange(n_pages, dtype=torch.int32, device=dev)
        self.n_free = torch.tensor([n_pages], dtype=torch.int32, device=dev)
        self.length = torch.zeros(n_seqs, dtype=torch.int32, device=dev)

    def plan(self, n_new, n_tokens, rows_per_seq=0, node_depth=None):
        return self.ctx.kv_plan(self.length, n_new, self.table, self.held, self.free, self.n_free, n_tokens, rows_per_seq, node_depth)

    def release(self):
        self.length = torch.zeros_like(self.length)
        self.plan(self.length, 0)


def decode(ctx, model, prompts, steps, trees, ngram=4, draft_len=4, max_cands=4, capacity=400):
    """Greedy decoding, ``steps`` model passes after the prompts'.  Returns the sequences (lists) and
    the cache, whose last tokens the next pass would store."""
    dev, B = ctx.device, len(prompts)
    lens = torch.tensor([p.numel() for p in prompts], dtype=torch.int32)
    offs = torch.cat([torch.zeros(1, dtype=torch.int32), lens.cumsum(0).to(torch.int32)]).to(dev)
    ids = torch.cat(prompts).to(torch.int32).to(dev)
    hist_offsets = (torch.arange(B + 1, dtype=torch.int32) * capacity).to(dev)
    hist = torch.full((B * capacity,), binding.NONE, dtype=torch.int32, device=dev)
    for b, p in enumerate(prompts):
        hist[b * capacity:b * capacity + p.numel()] = p.to(dev)
    hist_len, prompt_len = lens.to(dev), lens.to(dev)
    need = (capacity + 1 + max_cands * draft_len + PAGE - 1) // PAGE
    cache = Cache(model, B, B * need, need)

    # the prompts: one packed pass, the alignment table, each sequence's first token
    plan = cache.plan(prompt_len, ids.numel())
    logits = model(cache, ids, plan)
    align = ctx.align_sample(logits, ids, offs, k_extra=2)
    cache.length = plan["kv_len"]
    last = (offs[1:] - 1).long()
    ctx.append(hist, hist_offsets, hist_len, align["top1"][last].view(B, 1).contiguous(), torch.ones_like(hist_len))

    one = torch.ones_like(hist_len)
    slot = torch.arange(1 + max_cands * draft_len, device=dev)
    align_row_offsets = offs[:-1].contiguous()
    for _ in range(steps):
        root = hist[hist_offsets[:-1].long() + hist_len.long() - 1]     # emitted, but not in the cache yet
        if trees:
            d = ctx.draft(hist, hist_offsets, hist_len, prompt_len, ngram, draft_len, max_cands, align_ids=align["align_ids"],
                          align_n=align["n_extra"], align_row_offsets=align_row_offsets)
            t = ctx.tree_build(d["draft_ids"], d["draft_flags"], d["cand_len"], d["n_cands"])
            used = slot < t["n_nodes"][:, None]                         # the nodes in use, packed
            token, parent, flags, depth = (t["node_" + k][used] for k in ("token", "parent", "flags", "depth"))
            plan = cache.plan(t["n_nodes"], token.numel(), 0, depth)
            offsets = plan["tok_offsets"]
            tokens = token.clone()
            tokens[offsets[:-1].long()] = root
            logits = model(cache, tokens, plan, 0, parent)
            v = ctx.verify_tree(logits, token, parent, offsets, draft_len + 1, flags, mode=binding.VERIFY_STRICT_GREEDY)
            cache.length = ctx.kv_commit(cache.pages, cache.table, cache.length, plan["kv_len"], v["best_node"], parent, offsets)
            ctx.append(hist, hist_offsets, hist_len, v["emit_ids"], v["n_emit"])
        else:
            plan = cache.plan(one, B, 1)
            logits = model(cache, root, plan, 1)
            cache.length = plan["kv_len"]
            ctx.append(hist, hist_offsets, hist_len, logits.argmax(-1).to(torch.int32).view(B, 1), one)
    n = hist_len.tolist()
    return [hist[b * capacity:b * capacity + n[b]].tolist() for b in range(B)], cache


def prompts_for(n_seqs, vocab, seed=0):
    """Random tokens, repeated, so that there is something to draft from the start."""
    g = torch.Generator().manual_seed(seed)
    return [torch.randint(vocab, (7 + 5 * b,), generator=g).repeat(2 + b % 3).to(torch.int32) for b in range(n_seqs)]


def main():
    torch.backends.cuda.matmul.allow_tf32 = False
    ctx = binding.Context()
    model = Model(ctx)
    prompts = prompts_for(6, model.vocab)
    steps = 40
    fast, cache = decode(ctx, model, prompts, steps, trees=True)
    slow, _ = decode(ctx, model, prompts, max(len(s) - p.numel() for s, p in zip(fast, prompts)) - 1, trees=False)
    cache.release()
    for b, p in enumerate(prompts):
        n = len(fast[b]) - p.numel()
        print(f"sequence {b}: prompt {p.numel()}, {n} tokens in {steps + 1} passes, "
              f"as one by one: {fast[b] == slow[b][:len(fast[b])]}")
    print(f"status {ctx.poll_status()}, free pages {cache.n_free.item()} of {cache.free.numel()}")


if __name__ == "__main__":
    main()
