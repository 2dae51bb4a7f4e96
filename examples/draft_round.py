"""One draft round of a one-layer drafter, prompt to kept tree: the attention's calls and the trimmed head's together.

    prompt  ── qkv_to_cache ──▶ cache          (norm, rotation, keys and values of all tokens but the newest)
    level   ── qkv_to_cache, paged_attention, draft_tree_level ──▶ next frontier      (depth times)
    end     ── tree_rerank ──▶ the nodes kept for the target to verify

A level's nodes go into the cache behind the prompt, in the order they were drafted; each sees the prompt, its ancestors and
itself, by a mask over the last 64 cached tokens.  Weights are random (there is no checkpoint here); dense products are torch's.
The cache may be held in 8 or 4 bits; a layer may have a sliding window, with some first tokens that stay visible.

    python examples/draft_round.py [--cache e4m3 | e2m1] [--prompt 2000] [--window 512 --sinks 4]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2506_22694_amd as vt  # noqa: E402


class Drafter:
    """One decoder layer's attention and a trimmed head over `vocabulary` tokens, in bfloat16."""

    def __init__(self, d=1024, q_heads=8, kv_heads=4, head_dim=128, vocabulary=32000, trimmed=8192, seed=0, device="cuda",
                 window=None, sinks=0):
        g = torch.Generator(device=device).manual_seed(seed)

        def randn(*shape, std=1.0):
            return (torch.randn(shape, generator=g, device=device) * std).bfloat16()
        self.q_heads, self.kv_heads, self.head_dim = q_heads, kv_heads, head_dim
        self.window, self.sinks = window, sinks
        self.embedding = randn(vocabulary, d)
        self.qkv = randn(d, (q_heads + 2 * kv_heads) * head_dim, std=d ** -0.5)
        self.out = randn(q_heads * head_dim, d, std=(q_heads * head_dim) ** -0.5)
        self.q_norm, self.k_norm = (randn(head_dim, std=0.1) + 1 for _ in range(2))
        self.rope = vt.rope_table(8192, head_dim, 10000.0, device)
        counts = torch.randint(0, 1 << 20, (vocabulary,), generator=g, device=device)
        self.map, self.head = vt.build_trimmed_head(counts, randn(vocabulary, d, std=0.02), trimmed)

    def project(self, x):
        """q, k, v [n, heads, head_dim] of rows x: views of one product."""
        return torch.split((x @ self.qkv).unflatten(1, (-1, self.head_dim)), [self.q_heads, self.kv_heads, self.kv_heads], dim=1)

    def layer(self, tokens, cache, slots, positions, page_table, lengths, ws, max_length, row_start=None, tail_mask=None):
        """Hidden rows of new tokens of one request, whose keys and values go to `slots`."""
        x = self.embedding[tokens]
        q, k, v = self.project(x)
        q = vt.qkv_to_cache(q, k, v, cache, slots, positions, self.rope, self.q_norm, self.k_norm)
        a = vt.paged_attention(q, cache, page_table, lengths, row_start=row_start, max_rows=None if row_start is None else tokens.numel(),
                               tail_mask=tail_mask, max_length=max_length, ws=ws, window=self.window, sinks=self.sinks,
                               positions=positions if tail_mask is not None and self.window is not None else None)
        return x + a.flatten(1) @ self.out


class Memory:
    """What a program keeps from one round to the next: the calls' workspaces and a tree's memory."""

    def __init__(self, drafter, most_tokens, depth=3, width=8, keep=32, device="cuda"):
        k, d = drafter.head.shape
        self.depth, self.width, self.keep = depth, width, min(keep, depth * width)
        self.attend = vt.AttentionWorkspace(width, drafter.q_heads, drafter.kv_heads, drafter.head_dim, 1, width, most_tokens + depth * width, device)
        self.step = vt.StepWorkspace(width, k, d, width, device)
        self.rows = torch.arange(0, width + 1, width, dtype=torch.int32, device=device)      # a level's rows are one request's
        self.ids = torch.empty(width, width, dtype=torch.int32, device=device)
        self.logp = torch.empty(width, width, device=device)

    def tree(self, device):
        """Memory of one tree: parents (rows of the level before), tokens, cumulative log-probabilities, a row to each level; kept nodes."""
        shape = (self.depth, self.width)
        return (torch.empty(shape, dtype=torch.int32, device=device), torch.empty(shape, dtype=torch.int32, device=device),
                torch.empty(shape, device=device), torch.empty(self.keep, dtype=torch.int32, device=device))


def draft_round(drafter, prompt, cache, page_table, depth=3, width=8, keep=32, memory=None):
    """Drafts a tree behind `prompt` (token ids of one request).  Returns a dict of the tree's nodes in the order they were
    drafted: token, parent (-1: the prompt), depth, cumulative log-probability, hidden row each was drafted from; and `kept`.
    `memory`: one that is kept, whose depth, width and keep hold."""
    dev, n = prompt.device, prompt.numel()
    memory = memory or Memory(drafter, n, depth, width, keep, dev)
    depth, width = memory.depth, memory.width
    parents, tokens, cums, kept = memory.tree(dev)
    one = torch.zeros((), dtype=torch.int64, device=dev)

    def slots_of(first, count):
        return cache.slots(page_table, one.expand(count), torch.arange(first, first + count, device=dev))
    lengths = torch.arange(n, n + depth * width, width, dtype=torch.int32, device=dev)      # cached tokens, with those of a level
    # the prompt but its newest token: for its keys and values only
    if n > 1:
        q, k, v = drafter.project(drafter.embedding[prompt[:-1]])
        vt.qkv_to_cache(q, k, v, cache, slots_of(0, n - 1), torch.arange(n - 1, device=dev), drafter.rope, drafter.q_norm, drafter.k_norm)
    hidden = drafter.layer(prompt[-1:], cache, slots_of(n - 1, 1), torch.arange(n - 1, n, device=dev), page_table, lengths[:1], memory.attend, n)

    drafted_from, frontiers = [], []
    frontier = torch.full((1,), -1, dtype=torch.int64, device=dev)      # node numbers of the rows of `hidden`
    cum = torch.zeros(1, device=dev)
    seen = torch.zeros(1, dtype=torch.int64, device=dev)                # of each frontier node: itself and its ancestors, a bit each
    for level in range(depth):
        rows = hidden.shape[0]
        vt.draft_tree_level(hidden, drafter.head, drafter.map, width, cum, width, ws=memory.step, out=(parents[level], tokens[level], cums[level]),
                            out_ids=memory.ids[:rows], out_logp=memory.logp[:rows])
        parent, cum, drafted = parents[level].long(), cums[level], level * width
        drafted_from.append(hidden[parent])
        frontiers.append(frontier[parent])
        frontier = torch.arange(drafted, drafted + width, device=dev)
        seen = seen[parent] | (1 << frontier)
        if level + 1 < depth:
            nodes = drafted + width
            mask = (seen << (64 - nodes)) | ((1 << (64 - nodes)) - 1)      # bit j: token n + nodes - 64 + j
            hidden = drafter.layer(tokens[level], cache, slots_of(n + drafted, width), torch.full((width,), n + level, device=dev), page_table,
                                   lengths[level + 1:level + 2], memory.attend, n + nodes, memory.rows, mask)
    vt.tree_rerank(cums.flatten(), memory.keep, out=kept)
    return {"token": tokens.flatten(), "parent": torch.cat(frontiers), "depth": torch.arange(depth, dtype=torch.int32, device=dev).repeat_interleave(width),
            "cum": cums.flatten(), "hidden": torch.cat(drafted_from), "kept": kept}


def main():
    p = argparse.ArgumentParser()
    types = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "e2m1": torch.float4_e2m1fn_x2}
    p.add_argument("--cache", choices=list(types), default="bf16")
    p.add_argument("--prompt", type=int, default=1000)
    p.add_argument("--window", type=int)
    p.add_argument("--sinks", type=int, default=0)
    a = p.parse_args()
    drafter = Drafter(window=a.window, sinks=a.sinks)
    page = 64
    pages = -(-(a.prompt + 64) // page)
    cache = vt.KVCache(pages, page, drafter.kv_heads, drafter.head_dim, types[a.cache])
    page_table = torch.randperm(pages, device="cuda").int()[None].contiguous()
    prompt = torch.randint(0, 32000, (a.prompt,), device="cuda")
    tree = draft_round(drafter, prompt, cache, page_table)
    for i in tree["kept"].tolist():
        print(f"node {i:2d}  parent {tree['parent'][i].item():2d}  token {tree['token'][i].item():5d}  log-probability {tree['cum'][i].item():.3f}")


if __name__ == "__main__":
    main()
