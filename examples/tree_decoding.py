"""Greedy decoding of a toy model by drafted trees: the low-rank head, the paged cache and tree attention as a serving loop calls them.

The target is one attention layer with the low-rank head; the drafter is the same head on the embeddings alone.  Every step drafts a
tree of ten tokens for every sequence (the last token, three candidates after it, two after each of them), runs the target over all
trees at once, accepts the longest path that the target itself would have taken, and keeps its keys and values in the cache.  Nothing
in the loop waits for the GPU: what a step accepts stays on it.

    python examples/tree_decoding.py [--steps 20] [--sequences 4]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_10453_amd import binding  # noqa: E402

D_MODEL, Q_HEADS, KV_HEADS, HEAD_DIM, RANK, VOCAB, PAGE = 256, 4, 2, 64, 32, 8192, 16
WIDTHS = (3, 2)                                             # children of the last token, and of each of them
# the tree, the same for every sequence and step: node 0 is the last token, the committed context's only child
PARENTS = [-1, 0, 0, 0, 1, 1, 2, 2, 3, 3]


class Toy:
    """Random weights of the toy target (bf16): embedding, projections, and the low-rank head's A and B."""

    def __init__(self, seed: int = 0, device: str = "cuda"):
        g = torch.Generator().manual_seed(seed)
        def draw(rows, cols, scale):
            return (torch.randn(rows, cols, generator=g) * scale).to(torch.bfloat16).to(device)
        self.embedding = draw(VOCAB, D_MODEL, 1.0)
        self.qkv = draw(D_MODEL, (Q_HEADS + 2 * KV_HEADS) * HEAD_DIM, 2 * D_MODEL ** -0.5)
        self.out = draw(Q_HEADS * HEAD_DIM, D_MODEL, (Q_HEADS * HEAD_DIM) ** -0.5)
        self.A = draw(D_MODEL, RANK, D_MODEL ** -0.5)
        self.B = draw(RANK, VOCAB, 1.0)


def forward(model: Toy, cache, tokens, slots, first, mask):
    """The target's hidden rows for new tokens [n * T]; their keys and values go to the cache."""
    x = model.embedding[tokens]
    qkv = (x @ model.qkv).view(-1, Q_HEADS + 2 * KV_HEADS, HEAD_DIM)
    k, v = qkv[:, Q_HEADS:Q_HEADS + KV_HEADS], qkv[:, Q_HEADS + KV_HEADS:]
    binding.cache_append(cache, 0, k, v, slots, first)
    attended, _ = binding.tree_attention(cache, 0, qkv[:, :Q_HEADS], slots, first, mask=mask, lse=False)
    return x + attended.view(-1, Q_HEADS * HEAD_DIM) @ model.out


def draft(model: Toy, last):
    """A tree of tokens after the last one of every sequence, [n, 10]: the head on embeddings alone, level by level."""
    n, level, tokens = last.shape[0], last.view(-1, 1), [last.view(-1, 1)]
    for width in WIDTHS:
        ids, _ = binding.slimspec_head_topk(model.embedding[level.reshape(-1)].contiguous(), model.A, model.B, width)
        level = ids.long().view(n, -1)
        tokens.append(level)
    return torch.cat(tokens, 1)


def accept(tokens, chosen):
    """The path from node 0 that the target's own choices follow: (path [n, 3], how many nodes of it, the choice after it)."""
    n = tokens.shape[0]
    rows = torch.arange(n, device=tokens.device)
    path = torch.zeros((n, 3), dtype=torch.int64, device=tokens.device)
    count = torch.ones(n, dtype=torch.int64, device=tokens.device)
    node, follows = torch.zeros_like(count), torch.ones(n, dtype=torch.bool, device=tokens.device)
    parents = torch.tensor(PARENTS, device=tokens.device)
    for depth in (1, 2):
        hit = (parents[None] == node[:, None]) & (tokens == chosen[rows, node][:, None])
        found, child = hit.max(1)
        follows = follows & found
        node = torch.where(follows, child, node)
        path[:, depth] = node
        count += follows.long()
    return path.int(), count.int(), chosen[rows, node]


def prompt(sequences: int, length: int, seed: int, device: str = "cuda"):
    return torch.randint(0, VOCAB, (sequences, length), generator=torch.Generator().manual_seed(seed)).to(device)


def run(steps: int = 20, sequences: int = 4, seed: int = 0, prompt_length: int = 37):
    """Decodes; half way sequence 0 is forked into one more slot.  Returns the model and every slot's tokens (prompt first)."""
    model, n, T = Toy(seed), sequences, len(PARENTS)
    cache = binding.PagedCache.empty(1, (n + 1) * 40, KV_HEADS, PAGE, HEAD_DIM, slots=n + 1, slot_pages=40)
    i32 = dict(dtype=torch.int32, device="cuda")
    start = prompt(n, prompt_length, seed + 1)
    # the prompt but its last token, as a chain
    slots, first = torch.arange(n, **i32), torch.arange(n + 1, **i32) * (prompt_length - 1)
    reports = [binding.cache_reserve(cache, slots, first)]
    forward(model, cache, start[:, :-1].reshape(-1), slots, first, None)
    binding.cache_set_lens(cache, slots, torch.full((n,), prompt_length - 1, **i32))
    last, produced = start[:, -1], []
    for step in range(steps):
        if step == steps // 2:
            reports.append(binding.cache_fork(cache, torch.zeros(1, **i32), torch.full((1,), n, **i32)))
            slots, last = torch.arange(n + 1, **i32), torch.cat([last, last[:1]])
        m = slots.shape[0]
        first = torch.arange(m + 1, **i32) * T
        tokens = draft(model, last)
        mask = binding.tree_mask(torch.tensor(PARENTS * m, **i32), first, 1)
        reports.append(binding.cache_reserve(cache, slots, first))
        hidden = forward(model, cache, tokens.reshape(-1), slots, first, mask)
        chosen, _ = binding.slimspec_head_topk(hidden.contiguous(), model.A, model.B, 1)
        path, count, last = accept(tokens, chosen.long().view(m, T))
        lens = binding.cache_compact(cache, slots, first, path, count)
        binding.cache_set_lens(cache, slots, lens)
        produced.append((tokens, path, count, last))
    # the first wait: tokens of every slot, from what the steps accepted
    assert all(r.item() == 0 for r in reports), "the pool has no pages left"
    text = start.tolist() + [None]
    for step, (tokens, path, count, last) in enumerate(produced):
        if step == steps // 2:
            text[n] = list(text[0])
        for i in range(tokens.shape[0]):
            text[i] += [tokens[i, path[i, j]].item() for j in range(1, count[i].item())] + [last[i].item()]
    return model, text


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--sequences", type=int, default=4)
    a = ap.parse_args()
    _, text = run(a.steps, a.sequences)
    for i, t in enumerate(text):
        what = "fork of sequence 0" if i == a.sequences else f"sequence {i}"
        print(f"{what}: {len(t) - 37} tokens after the prompt in {a.steps} steps, the last ones {t[-5:]}")


if __name__ == "__main__":
    main()
