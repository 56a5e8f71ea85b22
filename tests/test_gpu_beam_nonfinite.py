"""The beam selection where a logit is not finite: each kind alone, of a live beam and of one that is not."""

from __future__ import annotations

import numpy as np
import pytest

from tests.test_gpu_beam import check_select
from tests.test_gpu_kv8 import BF16, F32, ops, rnd, torch  # noqa: F401

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("what", [NAN, INF, None])
def test_each_kind_of_logit_that_is_not_finite(ops, dtype, what):
    """In a live beam, alone: in a first or last block, a whole one, among words that are all out; and
    none of it (minus infinity alone)."""
    rng = np.random.default_rng(17)
    vocab = 2501
    for off in (0, 1, 3):
        for at in (0, 1, 700, 2048, 2499, 2500):
            for alone in (False, True):
                wide = rnd(rng, 8, vocab + 8, dtype=dtype, scale=2.0)
                z = wide[:, off:off + vocab]
                if alone:
                    z[5, max(0, at - 1200):at + 1200] = -INF
                z[5, at] = -INF if what is None else what
                got = check_select(ops, z, torch.full((2, 4), -2.0, device="cuda"), 6)
                bad = what is not None
                assert got[0][0].isfinite().all() and bool(got[0][1].isnan().all()) == bad
                assert bool((got[1][1] == -1).all()) == bad and bool((got[2][1] == -1).all()) == bad
                # the same in a beam that is not alive
                c = torch.tensor([[-2.0] * 4, [-2.0, -INF, -2, -2]], device="cuda")
                assert check_select(ops, z, c, 6)[0].isfinite().all()
