"""The beam selection's scores next to zero, and next to each other.

Tolerances.  A row's sum is at least 1, its likeliest word's.  An addition to a sum below 2^m is off by up
to 2^(m - 53): of 16 elements in a lane, 6 between the lanes of a unit, 6 + 16 between the units, and the
rescaling of a unit's sum, 2 in all: 46 2^-53 of the sum, and with 2^-52 of each exponential 48 2^-53 of it,
which the logarithm takes over as they are.  Where the other words are few next to 1 nothing else counts
(the logarithm is right to a step of its own, small, value): 48 2^-53.  For numbers up to 16 the logarithm adds a
step of 2^-49 and the score's three roundings 2^-50 each: below 2^-46 in all.  Then half a step of fp32."""

from __future__ import annotations

import math

import numpy as np
import pytest

from tests.test_gpu_kv8 import BF16, F32, f64, ops, rnd, torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [2, 500, 50257])
def test_scores_of_near_certain_words(ops, dtype, vocab):
    """One likely word, the others' odds e^-4 to e^-32: minus what they add up to, and never above zero."""
    odds = [-4.0, -8, -16, -20, -24, -28, -32]
    z = torch.empty(len(odds), vocab, dtype=dtype, device="cuda")
    for i, o in enumerate(odds):
        z[i] = o - math.log(max(vocab - 1, 1))
        z[i, (i * 97) % vocab] = 0.0
    s, p, v = ops.beam_select(z, torch.zeros(len(odds), 1, device="cuda"), 1)
    assert v[:, 0].tolist() == [(i * 97) % vocab for i in range(len(odds))]
    for i, (got, row) in enumerate(zip(f64(s)[:, 0], f64(z))):
        rest = math.fsum(math.exp(x) for x in row if x != 0.0)
        want = -math.log1p(rest)
        assert got <= 0 and abs(got - want) <= abs(want) * 2.0 ** -24 + 48 * 2.0 ** -53, (i, got, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [3, 1000, 50257, 152064])
def test_scores_in_64_bits(ops, dtype, vocab):
    """Beams whose scores so far all but cancel their best word's: what is left tells the sum's error."""
    rng = np.random.default_rng(vocab + 7)
    z = rnd(rng, 6, vocab, dtype=dtype, scale=2.0)
    x = z.float().cpu().numpy().astype(np.longdouble)
    top = x.max(1)
    lse = np.log(np.exp(x - top[:, None]).sum(1))
    c = lse.astype(np.float32)
    assert (lse < 16).all()
    s, p, v = ops.beam_select(z, torch.from_numpy(c)[:, None].cuda(), 1)
    want = (c.astype(np.longdouble) - lse).astype(np.float64)
    assert np.all(np.abs(f64(s)[:, 0] - want) <= 2.0 ** -46 + np.abs(want) * 2.0 ** -24)
