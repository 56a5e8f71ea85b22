"""A beam search's selection and the reordering of paged caches, in float64 and Python integers.
TEST INFRASTRUCTURE ONLY (nothing on the product path imports this).
"""

from __future__ import annotations

import numpy as np


def beam_select(logits, scores, k):
    """One search: logits [beams, vocab], scores [beams] -> (scores, parents, words) of the k best
    continuations, equal ones by the lowest (beam, word)."""
    found = []
    for i, c in enumerate(np.asarray(scores, np.float64)):
        if c == -np.inf:
            continue
        z = np.asarray(logits[i], np.float64)
        if np.isnan(c) or c == np.inf or np.isnan(z).any() or (z == np.inf).any():
            return np.full(k, np.nan), np.full(k, -1), np.full(k, -1)
        top = z.max()
        if top == -np.inf:
            continue
        lse = np.log(np.exp(z - top).sum())
        best = np.lexsort((np.arange(len(z)), -z))[:k]
        found += [(-(c + ((z[v] - top) - lse)), i, r, int(v)) for r, v in enumerate(best) if z[v] > -np.inf]
    found = sorted(found)[:k]
    out = np.full(k, -np.inf), np.full(k, -1), np.full(k, -1)
    for r, (s, i, _, v) in enumerate(found):
        out[0][r], out[1][r], out[2][r] = -s, i, v
    return out


def beam_reorder(pools, table, parent, length, spare, page):
    """In place: pools (arrays whose first axis is the page), table [n beams, entries], spare."""
    n, beams = parent.shape
    old, was, n_pages = table.copy(), [p.copy() for p in pools], len(pools[0])
    for b in range(n):
        at = min(max(int(length[b * beams]), 0), table.shape[1] * page)
        full, tail = at // page, at % page
        for i in range(beams):
            p, s = int(parent[b, i]), b * beams + i
            if not 0 <= p < beams or p == i:
                continue
            src = b * beams + p
            table[s, :full] = old[src, :full]
            if not tail:
                continue
            if not 0 <= old[src, full] < n_pages:
                table[s, full] = old[src, full]
                continue
            if 0 <= spare[s] < n_pages:
                for now, before in zip(pools, was):
                    now[spare[s]] = before[old[src, full]]
            table[s, full], spare[s] = spare[s], old[s, full]
