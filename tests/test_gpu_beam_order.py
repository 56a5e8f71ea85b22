"""The beam selection's order of beams that are alike: of equal scores the lowest beam's comes first, wherever
the rows lie."""

from __future__ import annotations

import numpy as np
import pytest

from tests.test_gpu_beam import check_select
from tests.test_gpu_kv8 import BF16, F32, ops, rnd, torch  # noqa: F401

pytestmark = pytest.mark.gpu
NAN = float("nan")


def in_turn(got, beams):
    """Of beams that are alike: each word for every beam, the lowest first."""
    s, p, v = (x.cpu().numpy() for x in got)
    k = p.shape[1]
    assert (p == np.arange(k) % beams).all(), p
    for j in range(0, k, beams):
        assert (v[:, j:j + beams] == v[:, j:j + 1]).all() and (s[:, j:j + beams] == s[:, j:j + 1]).all()


@pytest.mark.parametrize("vocab", [7, 1001, 7001, 30522, 32001, 50257])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_beams_that_are_alike_keep_their_order(ops, vocab, dtype):
    """Rows that follow each other without a gap start at every offset of 16 bytes."""
    for seed in range(4):
        rng = np.random.default_rng(100 * vocab + seed)
        z = rnd(rng, 1, vocab, dtype=dtype, scale=2.0).expand(8, vocab).contiguous()
        # (words of one logit each: a tie within a beam would be its next place)
        if vocab < 2000 and dtype == F32:
            in_turn(check_select(ops, z, torch.full((1, 8), -20.0, device="cuda"), min(56, 8 * vocab)), 8)
        check_select(ops, z, torch.full((2, 4), -20.0, device="cuda"), 32)
        check_select(ops, z, torch.full((1, 8), -20.0, device="cuda"), 64)


@pytest.mark.parametrize("vocab", [130, 7001, 32001])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_beams_that_are_alike_in_wider_rows(ops, vocab, dtype):
    """Every first offset, with rows an odd number of elements apart; rows that are alike up to a
    constant (logits and sums that are exact) have equal scores too."""
    rng = np.random.default_rng(vocab)
    for off in range(8):
        z = (rnd(rng, 1, vocab, dtype=F32, scale=32.0).round() / 16).clamp(-7, 7).to(dtype)
        wide = torch.full((8, vocab + off + 9 - (vocab + off) % 2), NAN, dtype=dtype, device="cuda")
        rows = wide[:, off:off + vocab]
        rows.copy_(z.expand(8, vocab))
        rows[1] += 4
        rows[6] -= 0.5
        assert wide.stride(0) % 2
        check_select(ops, rows, torch.full((2, 4), -3.0, device="cuda"), 32)
        check_select(ops, rows, torch.full((1, 8), -3.0, device="cuda"), 64)
