"""Attention over the 8-bit key-value cache at the ends of its range, against float64
(the stored rows by oracle/kv8.py) within the bound that tests/test_gpu_kv8.py derives."""

from __future__ import annotations

import numpy as np
import pytest

import oracle
from tests.test_gpu_kv8 import BF16, F32, Batch, f64, ints, ops, rnd, torch  # noqa: F401

pytestmark = pytest.mark.gpu

# Calls of every kernel: lengths, new rows (None: one each), KV heads, query heads a KV head,
# page-table entries beyond the contexts' (which shape the launch), page.
KERNELS = {
    "split_one": ([400, 33, 129], None, 2, 4, 0, 64),
    "split_several": ([1500, 700, 33], None, 1, 4, 90, 16),
    "split_rows": ([200, 90], [16, 7], 2, 2, 0, 16),
    "tile_64": ([70] * 26, [8] * 26, 8, 16, 0, 16),
    "tile_128": ([70] * 52, [8] * 52, 8, 16, 0, 16),
    "tile_several": ([700], [130], 4, 5, 2000, 128),
}


def store(bt, k, v):
    """Whole contexts k, v [sum of the lengths, n_kv, hd] appended; what they stand for, by sequence."""
    start = np.concatenate([[0], np.cumsum(bt.lens)])
    bt.cache.append(k, v, bt.length, row_start=ints(start.tolist()))
    return ([oracle.kv8_values(f64(x))[a:b] for a, b in zip(start, start[1:])] for x in (k, v))


def batch(ops, name, hd, seed):
    lens, rows, n_kv, G, extra, page = KERNELS[name]
    bt = Batch(ops, lens, rows, n_kv=n_kv, hd=hd, page=page, extra_pages=extra, seed=seed)
    return bt, n_kv * G


def attend(bt, q, **kw):
    return bt.cache.attend(q, bt.length, row_start=bt.row_start, max_rows=max(bt.rows), **kw)


def check(bt, q, out, K, V, scale, seen=None):
    """check_attend's bound (with `far`) on the GPU.  A row of zeros has no code of 127, but the
    scale of a largest value of 2^-60: where its weight is the largest, W <= 2^-60 / 127."""
    n_kv, hd = bt.n_kv, bt.hd
    G = q.shape[1] // n_kv
    single = q.dtype == BF16 and out.dtype == BF16
    for b, (n, r) in enumerate(zip(bt.lens, bt.rows)):
        at = slice(bt.start[b], bt.start[b] + r)
        k, v = (torch.from_numpy(x[b]).cuda().transpose(0, 1)[:, None].contiguous() for x in (K, V))
        qq = q[at].double().view(r, n_kv, G, hd).permute(1, 2, 0, 3).contiguous()
        x = qq @ k.transpose(-1, -2).contiguous() * scale
        pos = torch.arange(n, device="cuda")
        off = pos[None] > torch.arange(n - r, n, device="cuda")[:, None]
        if seen is not None:
            off = off | ~seen(pos)[None]
        x = x.masked_fill(off, float("-inf"))
        p = (x - x.amax(-1, keepdim=True)).exp()    # (softmax() drops what is below fp32's range)
        p /= p.sum(-1, keepdim=True)
        want, mag = p @ v, p @ v.abs()
        dots = (qq.abs() @ k.abs().transpose(-1, -2).contiguous()).amax(-1, keepdim=True) * abs(scale)
        e = (48 * 2.0 ** -24 + (0 if single else 2.0 ** -22)) * dots + 2.0 ** -20
        rel = 2 * e + (2.0 ** -11 if single else 2.0 ** -22) + (64 + n / 16) * 2.0 ** -24
        tol = mag * rel + want.abs() * torch.finfo(out.dtype).eps / 2 + 1e-30 + \
            n * 2.0 ** -31 * mag.amax(-1, keepdim=True).clamp(min=2.0 ** -60)
        err = (out[at].double().view(r, n_kv, G, hd).permute(1, 2, 0, 3) - want).abs()
        assert (err <= tol).all(), (b, float((err / tol).max()))


@pytest.mark.parametrize("length,entries", [(500, 34), (1090, 69), (40, 34)])
@pytest.mark.parametrize("hd", [64, 128])
def test_an_odd_number_of_partial_results(ops, hd, length, entries):
    """One row, one head, five or nine splits: five or nine outputs and states in the workspace."""
    bt = Batch(ops, [length], n_kv=1, hd=hd, page=16, extra_pages=entries - -(-length // 16))
    K, V = bt.fill()
    for dtype in (BF16, F32):
        q = rnd(bt.rng, 1, 1, hd, dtype=dtype)
        need = bt.cache.attend_workspace(1, 1, 1)
        assert need // 4 // hd % 2 == 1
        space = torch.full((need + 16,), 255, dtype=torch.uint8, device="cuda")
        check(bt, q, attend(bt, q, workspace=space[:need]), K, V, hd ** -0.5)
        assert (space[need:] == 255).all()


# ------------------------------------------------------------------ values' scales
@pytest.mark.parametrize("order", ["small_first", "large_first", "in_turn", "shuffled"])
@pytest.mark.parametrize("size", [1e4, 1e20, 1e30, 1e38])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("name", ["split_one", "split_several", "split_rows", "tile_several"])
def test_rows_of_zeros_beside_large_values(ops, name, hd, size, order):
    """Half the value rows zero (their scale is 2^-67), half about `size`, all of similar weight: the
    zero rows count in the softmax's sum whatever the scales and wherever they are."""
    bt, heads = batch(ops, name, hd, seed=11)
    n = sum(bt.lens)
    k, v = (rnd(bt.rng, n, bt.n_kv, hd, dtype=F32).clamp(-2.5, 2.5) for _ in "kv")
    at = np.concatenate([np.arange(m) for m in bt.lens])
    of = np.concatenate([np.full(m, m) for m in bt.lens])
    big = {"small_first": at >= of // 2, "large_first": at < of // 2, "in_turn": at // 32 % 2 == 1,
           "shuffled": bt.rng.random(n) < 0.5}[order]
    v *= torch.from_numpy(np.where(big, size, 0.0)).float().cuda()[:, None, None]
    K, V = store(bt, k, v)
    for dtype in (BF16, F32):
        q = rnd(bt.rng, bt.n_rows, heads, hd, dtype=dtype, scale=0.3)
        out = attend(bt, q)
        assert out.isfinite().all()
        check(bt, q, out, K, V, hd ** -0.5)


@pytest.mark.parametrize("size", [1e9, 1e34, 3e38])
@pytest.mark.parametrize("name", ["split_several", "tile_several"])
def test_many_small_weights_beside_a_large_one(ops, name, size):
    """One position of score s, all others of s - 8.5 (a weight of 2^-12 each, most of the sum
    together), with values of any size: none is lost from the sum or the output."""
    hd = 128
    bt, heads = batch(ops, name, hd, seed=12)
    n = sum(bt.lens)
    k = torch.zeros(n, bt.n_kv, hd, device="cuda")
    k[:, :, 0] = -8.5
    start = np.concatenate([[0], np.cumsum(bt.lens)])
    k[torch.from_numpy(start[:-1] + np.array(bt.lens) // 3).cuda(), :, 0] = 8.5
    v = rnd(bt.rng, n, bt.n_kv, hd, dtype=F32).clamp(-1, 1) * size
    K, V = store(bt, k, v)
    for dtype in (BF16, F32):
        q = torch.zeros(bt.n_rows, heads, hd, dtype=dtype, device="cuda")
        q[:, :, 0] = 0.5
        check(bt, q, attend(bt, q, scale=1.0), K, V, 1.0)


@pytest.mark.parametrize("name", list(KERNELS))
def test_scales_over_the_whole_range(ops, name):
    """Value rows from 2^-60 to 2^127 in any order, scores over some tens: weights, sums and
    output keep their precision where the largest values have the least weights and elsewhere."""
    for seed in range(4):
        bt, heads = batch(ops, name, 64, seed=20 + seed)
        n = sum(bt.lens)
        k, v = (rnd(bt.rng, n, bt.n_kv, 64, dtype=F32).clamp(-3, 3) for _ in "kv")
        size = 2.0 ** bt.rng.uniform(-60, 125, n)
        size[bt.rng.random(n) < 0.2] = 0.0
        v *= torch.from_numpy(size).float().cuda()[:, None, None]
        k *= [1.0, 6.0, 1.0, 40.0][seed]
        if seed == 2:    # the larger the value the lower the score
            k[:, :, 5] = torch.from_numpy(-np.log(np.maximum(size, 2.0 ** -60)) / 3).float().cuda()[:, None]
        K, V = store(bt, k, v)
        for dtype in (BF16, F32):
            q = rnd(bt.rng, bt.n_rows, heads, 64, dtype=dtype)
            if seed == 2:
                q[:, :, 5] = 24.0      # (its eighth, the scale's, times a third of the logarithm)
            out = attend(bt, q)
            check(bt, q, out, K, V, 0.125)


# ------------------------------------------------------------------ scores of minus infinity
@pytest.mark.parametrize("name", list(KERNELS))
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_whose_every_score_is_minus_infinity(ops, name, dtype):
    """An infinite query over keys of the opposite sign, and finite queries whose scores pass the
    largest fp32: the quotient of two zeros, NaN; where nothing is seen zeros all the same, and
    finite scores beside such ones are attended alone."""
    hd = 64
    bt, heads = batch(ops, name, hd, seed=30)
    n = sum(bt.lens)
    k = torch.zeros(n, bt.n_kv, hd, device="cuda")
    v = rnd(bt.rng, n, bt.n_kv, hd, dtype=F32)
    q = torch.zeros(bt.n_rows, heads, hd, dtype=dtype, device="cuda")
    for value, size in ((float("inf"), 1.0), (1e30, 1e30)):
        for sign in (1.0, -1.0):
            k[:, :, 7] = -sign * size
            store(bt, k, v)
            q[:, :, 7] = sign * value
            out = attend(bt, q)
            assert out.isnan().all(), (value, sign)
            # the other sign: plus infinity less itself
            q[:, :, 7] = -sign * value
            assert attend(bt, q).isnan().all()
    # a sequence without positions or pages, beside others
    length, table = bt.length.clone(), bt.cache.table.clone()
    bt.length[-1] = 0
    if len(bt.lens) > 1:
        bt.cache.table[0] = -1
    q[:, :, 7] = 1e30
    k[:, :, 7] = -1e30
    start = np.concatenate([[0], np.cumsum(bt.lens)])
    bt.cache.append(k, v, length, row_start=ints(start.tolist()))
    out = attend(bt, q)
    for b in range(len(bt.lens)):
        got = out[bt.start[b]:bt.start[b + 1]]
        assert not got.any() if b == len(bt.lens) - 1 or b == 0 else got.isnan().all(), b
    bt.length.copy_(length), bt.cache.table.copy_(table)
    # every fifth position finite (a score of zero), the first of them position 0
    finite = np.concatenate([np.arange(m) % 5 == 0 for m in bt.lens])
    k[:, :, 7] = torch.from_numpy(np.where(finite, 0.0, -1e30)).float().cuda()[:, None]
    K, V = store(bt, k, v)
    out = attend(bt, q)
    check(bt, torch.zeros_like(q), out, [x * 0 for x in K], V, 0.125,
                 seen=lambda j: j % 5 == 0)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_of_one_position_and_scores_of_infinity(ops, dtype):
    """One, two and three positions: an infinite query element over a key element of either sign is
    NaN, for single tokens and for a prompt whose first row sees one position."""
    for rows in (None, [1, 2, 3]):
        bt = Batch(ops, [1, 2, 3], rows, n_kv=1, hd=128, page=16, seed=31)
        v = rnd(bt.rng, 6, 1, 128, dtype=F32)
        k = torch.ones_like(v)
        for sign in (1.0, -1.0):
            k[:, :, 9] = sign
            store(bt, k, v)
            for inf in (float("inf"), -float("inf")):
                q = rnd(bt.rng, bt.n_rows, 3, 128, dtype=dtype)
                q[:, 1, 9] = inf
                out = attend(bt, q)
                assert out[:, 1].isnan().all() and out[:, ::2].isfinite().all(), (rows, sign, inf)


# ------------------------------------------------------------------ the longest contexts
@pytest.mark.parametrize("rows", [None, 200])
def test_contexts_of_all_positions_that_32_bits_count(ops, rows):
    """2^31 - 1 positions (one page named 2^24 - 1 times, then another): the last page's positions
    have all but 2^31 e^-40 of the weight, and the slot past the end, of more, has none."""
    hd, page, n = 64, 128, 2 ** 31 - 1
    table = torch.zeros(1, 2 ** 24, dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    cache = ops.KvCache.empty(2, 1, hd, table, page=page)
    rng = np.random.default_rng(40)
    v = rnd(rng, 256, 1, hd, dtype=F32)
    k = torch.zeros_like(v)
    k[128:255, 0, 0], k[255, 0, 0] = 40.0, 45.0
    v[255] = 1000.0
    ops.KvCache(cache.pool, ints([[0, 1]]), page=page, head_dim=hd).append(
        k, v, ints([256]), row_start=ints([0, 256]))
    V = oracle.kv8_values(f64(v))[:, 0]
    r = rows or 1
    q = torch.zeros(r, 1, hd, device="cuda")
    q[:, 0, 0] = 1.0
    kw = {} if rows is None else dict(row_start=ints([0, rows]), max_rows=rows)
    out = f64(cache.attend(q, ints([n]), scale=1.0, **kw))[:, 0]
    for i in {0, r // 2, r - 5, r - 1} & set(range(r)):
        seen = V[128:256 - (r - i)] if r - i < 128 else None
        if seen is None:
            continue
        # the others: at most 2^31 e^-40 / len(seen) of the weight, each way; two fp16 terms, and
        # the sum of the last page's 127 weights
        tol = 2.0 ** 31 * np.exp(-40.0) * np.abs(V).max() * 2 + 2.0 ** -17 * np.abs(seen).mean(0)
        assert np.all(np.abs(out[i] - seen.mean(0)) <= tol), i
    if rows:
        # rows that do not see the last page: the plain mean of the first.  A lane's sum of 2^19
        # steps is off by at most 2^19 / 2 roundings of 2^-24 of it, a product's by twice that.
        first = V[:128].mean(0)
        assert np.all(np.abs(out[0] - first) <= 2.0 ** -4 * np.abs(V[:128]).mean(0))


# ------------------------------------------------------------------ the most rows
def test_as_many_rows_and_heads_as_a_call_takes(ops):
    """2^24 rows of one head, 2^15 in each of 512 sequences that share their pages: the last 600
    see their positions, the others nothing; split in two (hints of one row and 544
    positions), so that every row is merged."""
    n_seqs, r, n, hd = 512, 2 ** 15, 600, 64
    bt = Batch(ops, [n], [n], n_kv=1, hd=hd, page=16, seed=50)
    K, V = bt.fill()
    cache = ops.KvCache(bt.cache.pool, bt.table.expand(n_seqs, -1).contiguous(), page=16, head_dim=hd)
    start = torch.arange(n_seqs + 1, dtype=torch.int32, device="cuda") * r
    one = rnd(bt.rng, r, 1, hd)
    q = one.repeat(n_seqs, 1, 1)
    out = torch.full_like(q, 7.0)
    hints = dict(max_rows=1, max_length=544)
    assert cache.attend_workspace(n_seqs * r, 1, n_seqs, row_start=True, **hints) // (4 * n_seqs * r) \
        == 2 * (hd + 4)
    cache.attend(q, torch.full((n_seqs,), n, dtype=torch.int32, device="cuda"), row_start=start, out=out,
                 **hints)
    first = out[:r].clone()
    assert not first[:r - n].any()
    check(bt, one[r - n:], first[r - n:], K, V, hd ** -0.5)
    for b in range(n_seqs):
        assert torch.equal(out[b * r:(b + 1) * r], first), b
