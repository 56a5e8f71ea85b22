"""Attention over the 4-bit key-value cache at the ends of its range, and calls that its documents allow
and that are rarely made."""

from __future__ import annotations

import numpy as np
import pytest

import oracle
from tests.test_gpu_kv4 import Batch4, check_attend, sub_batch
from tests.test_gpu_kv8 import BF16, F32, f64, ints, ops, rnd, torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [None, 200])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_contexts_of_all_positions_that_32_bits_count(ops, rows, dtype):
    """2^31 - 1 positions (one page named 2^24 - 1 times, then another): the last page's positions
    have all but 2^31 e^-48 of the weight, and the slot past the end, of more, has none."""
    hd, page, n = 64, 128, 2 ** 31 - 1
    table = torch.zeros(1, 2 ** 24, dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    cache = ops.KvCache.empty(2, 1, hd, table, page=page, bits=4)
    rng = np.random.default_rng(40)
    v = rnd(rng, 256, 1, hd, dtype=F32)
    k = torch.zeros_like(v)
    k[128:255, 0, 0], k[255, 0, 0] = 48.0, 64.0      # (both are kept as they are)
    v[255] = 1000.0
    ops.KvCache(cache.pool, ints([[0, 1]]), page=page, head_dim=hd, bits=4).append(
        k, v, ints([256]), row_start=ints([0, 256]))
    V = oracle.kv4_values(f64(v))[:, 0]
    r = rows or 1
    q = torch.zeros(r, 1, hd, device="cuda", dtype=dtype)
    q[:, 0, 0] = 1.0
    kw = {} if rows is None else dict(row_start=ints([0, rows]), max_rows=rows)
    out = f64(cache.attend(q, ints([n]), scale=1.0, **kw))[:, 0]
    for i in {0, r // 2, r - 5, r - 1} & set(range(r)):
        seen = V[128:256 - (r - i)] if r - i < 128 else None
        if seen is None:
            continue
        # the others: at most 2^31 e^-48 / len(seen) of the weight, each way; a weight's terms (2^-11 of
        # it for bf16 rows), the sum of the last page's 127 weights, and the result's rounding
        tol = 2.0 ** 31 * np.exp(-48.0) * np.abs(V).max() * 2 + \
            (2.0 ** -11 if dtype == BF16 else 2.0 ** -17) * np.abs(seen).mean(0) + \
            np.abs(seen.mean(0)) * torch.finfo(dtype).eps / 2
        assert np.all(np.abs(out[i] - seen.mean(0)) <= tol), i
    if rows:
        # rows that do not see the last page: the plain mean of the first.  A lane's sum of 2^19
        # steps is off by at most 2^19 / 2 roundings of 2^-24 of it, a product's by twice that.
        first = V[:128].mean(0)
        assert np.all(np.abs(out[0] - first) <= 2.0 ** -4 * np.abs(V[:128]).mean(0))


@pytest.mark.parametrize("hints", [dict(max_rows=400, max_length=500), dict(max_rows=4, max_length=500),
                                   dict(max_rows=400, max_length=30000)])
def test_prompts_in_a_graph(ops, hints):
    """A packed batch of prompts (its rows padded) captured and replayed as rows, lengths and pages change
    in place, against eager calls."""
    rng = np.random.default_rng(12)
    H, G, hd, page = 4, 8, 128, 16
    table = ints(rng.permutation(96).reshape(2, 48).tolist())
    cache = ops.KvCache.empty(96, H, hd, table, page=page, bits=4)
    cache.pool.zero_()
    t = ops.rope_table(800, hd)
    q, k, v = (rnd(rng, 440, n, hd) for n in (H * G, H, H))
    length, start = ints([400, 40]), ints([0, 400, 440])
    qq, out = torch.empty_like(q), torch.empty_like(q)

    def step():
        cache.append(k, v, length, row_start=start, rope=t, q=q, q_out=qq)
        cache.attend(qq, length, row_start=start, out=out, **hints)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        step()
    for lens, rows in (((400, 40), (400, 40)), ((640, 200), (240, 160)), ((641, 768), (1, 436)),
                       ((641, 768), (0, 0)), ((700, 3), (59, 3))):
        length.copy_(ints(lens))
        start.copy_(ints([1, 1 + rows[0], 1 + sum(rows)]))
        for x in (q, k, v):
            x.copy_(rnd(rng, *x.shape))
        kept = cache.pool.clone()
        out.fill_(3), qq.fill_(3)
        step()
        want, pool = out.clone(), cache.pool.clone()
        cache.pool.copy_(kept)
        out.fill_(3), qq.fill_(3)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(cache.pool, pool)
        assert (out[0] == 3).all() and (out[1 + sum(rows):] == 3).all()


def test_many_sequences_in_a_part_of_a_wider_table(ops):
    """3000 sequences of none to three new rows each, in a table whose rows are longer than the cache's
    part of them."""
    rng = np.random.default_rng(31)
    n, H, G, hd, page = 3000, 1, 4, 64, 16
    new = rng.integers(0, 4, n)
    new[:5], new[-3:] = 0, 0
    lens = new + rng.integers(0, 20, n)
    wide = ints(rng.integers(-9, 0, (n, 9)).tolist())
    wide[:, 4:6] = ints(rng.permutation(2 * n).reshape(n, 2).tolist())
    cache = ops.KvCache.empty(2 * n, H, hd, wide[:, 4:6], page=page, bits=4)
    length = ints(lens.tolist())
    whole = np.concatenate([[0], np.cumsum(lens)])
    k, v = (rnd(rng, int(whole[-1]), H, hd) for _ in "kv")
    cache.append(k, v, length, row_start=ints(whole.tolist()))
    K, V = oracle.kv4_values(f64(k)), oracle.kv4_values(f64(v))
    start = np.concatenate([[0], np.cumsum(new)])
    for dtype in (BF16, F32):
        q = rnd(rng, int(start[-1]), H * G, hd, dtype=dtype)
        out = cache.attend(q, length, row_start=ints(start.tolist()))
        check_attend(sub_batch(lens.tolist(), new.tolist(), start), q, out,
                     [K[a:b] for a, b in zip(whole, whole[1:])], [V[a:b] for a, b in zip(whole, whole[1:])], 0.125)


def test_named_streams_and_memory_in_use(ops):
    """A cache dropped while a call on a named stream still waits stays allocated until that is done."""
    side = torch.cuda.Stream()
    x = torch.zeros(1, 2, 64, device="cuda")
    one = ints([1])
    for call in ("append", "read", "attend"):
        cache = ops.KvCache.empty(64, 2, 64, ints([[0]]), page=64, bits=4)
        kept, size = cache.pool.data_ptr(), cache.pool.numel()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(200_000_000)
        if call == "append":
            cache.append(x, x, one, stream=side)
        elif call == "read":
            cache.read(one, stream=side)
        else:
            cache.attend(x, one, stream=side)
        del cache
        new = torch.empty(size, dtype=torch.uint8, device="cuda")
        busy = not side.query()
        assert busy and new.data_ptr() != kept
        torch.cuda.synchronize()


def test_no_sequences(ops):
    cache = ops.KvCache.empty(2, 2, 64, torch.zeros(0, 3, dtype=torch.int32, device="cuda"), page=16, bits=4)
    none, x = ints([]).view(0), torch.zeros(0, 2, 64, device="cuda")
    assert cache.append(x, x, none) is None
    assert cache.attend(x, none).shape == (0, 2, 64) and cache.read(none)[0].shape == (0, 2, 64)


def test_single_words_of_a_padded_table(ops):
    """A batch of 1 and a table row of one entry; a page that ends with the context."""
    for n in (1, 16, 15):
        bt = Batch4(ops, [n], n_kv=1, hd=64, page=16, extra_pages=0)
        K, V = bt.fill()
        for dtype in (BF16, F32):
            q = rnd(bt.rng, 1, 1, 64, dtype=dtype)
            check_attend(bt, q, bt.cache.attend(q, bt.length), K, V, 0.125)
