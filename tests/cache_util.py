"""Plain forms of the paged cache's calls and of the attention over it, in 64 bits and Python lists (test-side only)."""
from __future__ import annotations

import numpy as np
import torch

# half the distance of neighbouring values, relative: a rounding to the type is off by at most this
ROUNDING = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def ancestor_sets(parents):
    """Of each token of one tree the set of itself and its ancestors."""
    sets = []
    for t, p in enumerate(parents):
        sets.append({t} | (sets[p] if 0 <= p < t else set()))
    return sets


def mask_words(sets, words):
    """Rows of 64-bit words (as int64) from sets of token indices."""
    rows = np.zeros((len(sets), words), dtype=np.uint64)
    for t, seen in enumerate(sets):
        for j in seen:
            if j < 64 * words:
                rows[t, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return torch.from_numpy(rows.view(np.int64))


def attention_reference(q, k, v, seen, scale):
    """Rows of one sequence and one key head in 64 bits, with bounds on what a kernel's row may be off by.

    q [rows, D], k, v [places, D] (float64, CPU), seen [rows, places] bool.  Returns out, lse, bound_out, bound_lse; the bounds follow from
    the roundings that the call's definition allows: scores and sums in 32 bits (a sum of D products is off by at most D 2^-24 times the
    sum of their sizes), the weights and the result rounded to the type once each.
    """
    rows, D = q.shape
    out, lse = torch.zeros(rows, D, dtype=torch.float64), torch.full((rows,), -np.inf, dtype=torch.float64)
    size, err = torch.zeros(rows, D, dtype=torch.float64), torch.zeros(rows, dtype=torch.float64)
    raw, count = torch.zeros(rows, D, dtype=torch.float64), torch.zeros(rows, dtype=torch.float64)
    for r in range(rows):
        at = seen[r].nonzero().view(-1)
        if not len(at):
            continue
        s = (k[at] @ q[r]) * scale
        lse[r] = torch.logsumexp(s, 0)
        w = torch.exp(s - lse[r])
        out[r], size[r], raw[r], count[r] = w @ v[at], w @ v[at].abs(), v[at].abs().sum(0), len(at)
        # the score's sum, its products with scale and log2 e, and the difference to the maximum
        err[r] = ((D + 8) * 2.0 ** -24 * abs(scale) * (k[at].abs() @ q[r].abs())).max() + 2.0 ** -22
    return out, lse, size, err, raw, count


def attention_bounds(out, lse, size, err, raw, count, dtype):
    u = ROUNDING[dtype]
    # weights of relative error e^(2 err) - 1 and u, sums in 32 bits of up to `count` terms in some order of at most 2^-24 each per step of a
    # chain no longer than count; the result rounded once.  fp16 weights below 2^-14 are off by up to 2^-25 each, values likewise.
    sums = (count.sqrt() + 64) * 2.0 ** -24 * 4
    bound = (u + 4 * err[:, None] + sums[:, None]) * size * 1.01 + u * (out.abs() + (u + 4 * err[:, None]) * size)
    if dtype == torch.float16:
        bound = bound + raw * 2.0 ** -25 + 2.0 ** -25
    bound_lse = 2 * err + sums + 2.0 ** -22 * lse.abs().nan_to_num(posinf=0, neginf=0) + 2.0 ** -22
    return bound + 1e-30, bound_lse


class Books:
    """The books of a cache as lists, and its rows by what was last written to a place: {(slot, place): tag}."""

    def __init__(self, pages, page_size, slots, slot_pages):
        self.P, self.slot_pages = page_size, slot_pages
        self.table = [[0] * slot_pages for _ in range(slots)]
        self.held, self.lens, self.refs = [0] * slots, [0] * slots, [0] * pages

    def _take(self, wanted):
        free = [p for p, r in enumerate(self.refs) if r == 0]
        return None if len(free) < wanted else free[:wanted], wanted - len(free)

    def reserve(self, slots, counts):
        need = []
        for s, t in zip(slots, counts):
            if not 0 <= s < len(self.lens) or t < 0 or -(-(self.lens[s] + t) // self.P) > self.slot_pages:
                return -1
            need.append(max(0, -(-(self.lens[s] + t) // self.P) - self.held[s]))
        pages, lacking = self._take(sum(need))
        if pages is None:
            return lacking
        for s, m in zip(slots, need):
            for _ in range(m):
                page = pages.pop(0)
                self.table[s][self.held[s]] = page
                self.refs[page] = 1
                self.held[s] += 1
        return 0

    def set_lens(self, slots, lens):
        for s, x in zip(slots, lens):
            x = min(max(x, 0), self.held[s] * self.P)
            while self.held[s] > -(-x // self.P):
                self.held[s] -= 1
                self.refs[self.table[s][self.held[s]]] -= 1
            self.lens[s] = x

    def fork(self, parents, children):
        for p, c in zip(parents, children):
            if not (0 <= p < len(self.lens) and 0 <= c < len(self.lens)) or p == c or self.held[c] or self.lens[p] > self.held[p] * self.P:
                return -1, []
        lens = [self.lens[p] for p in parents]
        pages, lacking = self._take(sum(1 for x in lens if x % self.P))
        if pages is None:
            return lacking, []
        copies = []
        for p, c, x in zip(parents, children, lens):
            full, rest = divmod(x, self.P)
            for j in range(full):
                self.table[c][j] = self.table[p][j]
                self.refs[self.table[p][j]] += 1
            if rest:
                self.table[c][full] = pages.pop(0)
                self.refs[self.table[c][full]] = 1
                copies.append((self.table[p][full], self.table[c][full], rest))
            self.held[c], self.lens[c] = full + (rest > 0), x
        return 0, copies
