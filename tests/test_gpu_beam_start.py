"""Beam searches that begin from a prompt whose last page is partial, over paged caches of both widths."""

from __future__ import annotations

import numpy as np
import pytest

import oracle
from tests.test_gpu_kv8 import F32, f64, ints, ops, rnd, torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("length", [5, 16, 37, 63])
def test_a_search_begins_from_a_prompt(ops, bits, length):
    """The prompt lies in its first beam's pages.  One reordering with every parent that beam shares the
    full pages and gives each beam a partial page of its own; then tokens and reorderings in turn: what a
    beam reads back is its own words throughout."""
    rng = np.random.default_rng(length + bits)
    n, beams, H, hd, page, steps = 2, 4, 2, 64, 16, 24
    seqs, entries = n * beams, 6
    values = oracle.kv4_values if bits == 4 else oracle.kv8_values
    table = ints(rng.permutation(seqs * entries).reshape(seqs, entries).tolist())
    spare = ints((seqs * entries + np.arange(seqs)).tolist())
    caches = [ops.KvCache.empty(seqs * (entries + 1), H, hd, table, page=page, bits=bits) for _ in range(2)]
    prompts = [ops.KvCache(c.pool, table[::beams], page=page, head_dim=hd, bits=bits) for c in caches]
    held = []                                            # of each layer: of each beam: rows of k, of v
    for c, first in zip(caches, prompts):
        c.pool.zero_()
        k, v = (rnd(rng, n * length, H, hd, dtype=F32) for _ in "kv")
        first.append(k, v, ints([length] * n), row_start=ints([length * b for b in range(n + 1)]))
        held.append([[f64(x[length * b:length * (b + 1)]) for x in (k, v)] for b in range(n)
                     for _ in range(beams)])
    at = length
    ops.beam_reorder(caches, ints([[0] * beams] * n), ints([at] * seqs), spare)
    for step in range(steps):
        # pages that can still be written belong to one beam alone, spares to none
        t = table.cpu().numpy()
        ends = t[:, at // page]
        assert len(set(ends) | set(spare.tolist())) == 2 * seqs
        for layer, c in enumerate(caches):
            rk, rv = c.read(ints([at] * seqs), row_start=ints((np.arange(seqs + 1) * at).tolist()),
                            n_rows=seqs * at, dtype=F32)
            for sq in range(seqs):
                for got, want in zip((rk, rv), held[layer][sq]):
                    assert np.array_equal(f64(got[sq * at:(sq + 1) * at]), values(want).astype(np.float32))
        at += 1
        parent = rng.integers(0, beams, (n, beams))
        for layer, c in enumerate(caches):
            k, v = (rnd(rng, seqs, H, hd, dtype=F32) for _ in "kv")
            c.append(k, v, ints([at] * seqs))
            new = [[np.concatenate([old, f64(x[sq:sq + 1])]) for old, x in zip(held[layer][sq], (k, v))]
                   for sq in range(seqs)]
            held[layer] = [new[b * beams + p] for b in range(n) for p in parent[b]]
        ops.beam_reorder(caches, ints(parent.tolist()), ints([at] * seqs), spare)
