"""Attention over the 4-bit cache where scores are too large for a reference to hold a shift, and where
values are so large that sums of them leave fp32."""

from __future__ import annotations

import numpy as np
import pytest

from tests.test_gpu_kv4 import Batch4, check_on_gpu
from tests.test_gpu_kv8 import BF16, F32, PLAN_CASES, ints, ops, rnd, torch  # noqa: F401

pytestmark = pytest.mark.gpu


def case(ops, n_seqs, rows, length, n_kv, G, hd, entries, page, values, **kw):
    """Contexts of one key throughout; `values` (positions) -> factors of normal values."""
    need = -(-length // page)
    bt = Batch4(ops, [length] * n_seqs, [rows] * n_seqs, n_kv=n_kv, hd=hd, page=page, seed=rows + n_seqs,
                extra_pages=entries - need)
    n = n_seqs * length
    k = rnd(bt.rng, 1, n_kv, hd, dtype=F32).expand(n, n_kv, hd).contiguous()
    v = rnd(bt.rng, n, n_kv, hd, dtype=F32)
    size = values(np.arange(n) % length).astype(np.float32)
    v *= torch.from_numpy(size).cuda()[:, None, None]
    return bt, *bt.store(k, v)


def check_alike(bt, q, K, V, **kw):
    """Equal scores weigh alike: as those of queries of zero."""
    out = bt.cache.attend(q, bt.length, row_start=bt.row_start, **kw)
    assert out.isfinite().all()
    check_on_gpu(bt, torch.zeros_like(q), out, K, V)


@pytest.mark.parametrize("n_seqs,rows,length,n_kv,G,hd,entries,page", PLAN_CASES + [(1, 200, 700, 4, 5, 64, 2100, 128)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_large_scores_beside_ordinary_ones(ops, n_seqs, rows, length, n_kv, G, hd, entries, page, dtype):
    """Tiles of 16 rows x heads of large queries in turn with ordinary ones, either first, and every
    other row: what a row's neighbours are does not matter."""
    bt, K, V = case(ops, n_seqs, rows, length, n_kv, G, hd, entries, page, lambda j: 1.0 + 0 * j)
    of_row = np.arange(n_seqs * rows) % rows
    place = of_row[:, None] * G + np.arange(n_kv * G) % G       # among the rows x heads of a KV head
    for pick in (place // 16 % 2 == 0, place // 16 % 2 == 1, place % 2 == 0):
        for size in (3e6, 3e7, 1.7e8):
            q = rnd(bt.rng, bt.n_rows, n_kv * G, hd, dtype=dtype)
            q *= torch.from_numpy(np.where(pick, size, 1.0).astype(np.float32)).cuda().to(dtype)[..., None]
            check_alike(bt, q, K, V, max_rows=rows)


@pytest.mark.parametrize("n_seqs,rows,length,n_kv,G,hd,entries,page",
                         PLAN_CASES + [(3, 1, 3000, 2, 2, 64, 190, 16), (3, 1, 3000, 2, 2, 128, 190, 16)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_large_values_midway_under_large_scores(ops, n_seqs, rows, length, n_kv, G, hd, entries, page, dtype):
    """Ordinary values first, ones past 2^100 and to fp32's end later: the positions before them weigh what
    they did."""
    for late, big in ((1 - rows / length / 2, 2.0 ** 101), (0.7, 2.0 ** 124)):
        bt, K, V = case(ops, n_seqs, rows, length, n_kv, G, hd, entries, page,
                        lambda j: np.where(j >= late * length, big, 1.0))
        for size in (1.0, 3e6, 2.0 ** 28, 1e9, 3e10):
            q = rnd(bt.rng, bt.n_rows, n_kv * G, hd, dtype=dtype) * size
            check_alike(bt, q, K, V, max_rows=rows)


@pytest.mark.parametrize("rows", [None, 200])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lg,exponent", [(21, 99), (27, 99), (28, 125)])
def test_long_contexts_of_large_values(ops, rows, dtype, lg, exponent):
    """2^lg positions that all hold +-6 2^exponent, the first page with scores 4.9 ln 2 below the others' or
    all with the same: their mean, though fp32 does not hold their sum.  A lane adds at most 2^28 / (32 x
    128) = 2^16 times to each of its two sums, each time within 2^-24: 2^-7 in all."""
    hd, page, n = 64, 128, 2 ** lg
    table = torch.ones(1, n // page, dtype=torch.int32, device="cuda")
    table[0, 0] = 0
    cache = ops.KvCache.empty(2, 1, hd, table, page=page, bits=4)
    k = torch.zeros(256, 1, hd, device="cuda")
    k[128:, 0, 0] = 4.0
    v = torch.full((256, 1, hd), 6 * 2.0 ** exponent, device="cuda")
    v[:, :, 1::2] *= -1
    ops.KvCache(cache.pool, ints([[0, 1]]), page=page, head_dim=hd, bits=4).append(
        k, v, ints([256]), row_start=ints([0, 256]))
    r = rows or 1
    q = torch.zeros(r, 1, hd, device="cuda", dtype=dtype)
    q[:, 0, 0] = 1.0
    kw = {} if rows is None else dict(row_start=ints([0, rows]), max_rows=rows)
    for scale in (0.0, 4.9 * np.log(2.0) / 4):
        out = cache.attend(q, ints([n]), scale=scale, **kw).double()
        want = v[0].double()
        assert ((out - want).abs() <= want.abs() * (2.0 ** -7 + 2.0 ** -8)).all()
