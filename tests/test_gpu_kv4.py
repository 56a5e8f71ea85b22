"""The 4-bit key-value cache and attention over it, against their definitions in float64
(oracle/kv4.py).

Tolerances.  Codes, scales and rotations have one right answer and are compared for equality (a
bf16 result with the rounding of that answer).  Attention: with S the largest sum |q_d k_d| scale
of a row and A the output with |v| in place of v, a score is off by at most e = 64 2^-24 S + 2^-20
(a sum of 128 products in fp32, with the roundings of a third bf16 term of the query, of the
factor and of the difference; the exponential's argument and result), which moves a weight and the
sum by e each; a weight is off by at most 2^-24 of itself (three bf16 terms), for bf16 rows 2^-11 (one
fp16 term; two bf16 terms where the values' scales do not fit fp16: 2^-16) or 2^-31 of the row's largest
weight (half of fp16's least step, 2^-24, with that at 2^6 or more: n 2^-31 of the largest |v| at most
in all); the sums over n positions add at most (64 + n / 16) roundings of
2^-24 A, and those of several terms as many again; and the result is rounded once, by eps / 2 of
itself.  Weights are fp32 (and their terms bf16) with the largest at 1 or more: one below 2^-126, or a
term below it, may count as zero, which is off by at most 2^-126 |v| a position and term, of a sum
of at least 1: 3 n 2^-126 of the largest |v| that the row sees.  Rows that have met values of 2^100
hold their largest weight at 2^-32 (what is summed would else leave fp32), and 2^-126 is 2^-94 of it."""

from __future__ import annotations

import numpy as np
import pytest

import oracle
from tests.test_gpu_kv8 import BF16, F32, PLAN_CASES, SHAPES, Batch, f64, ints, ops, rnd  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


class Batch4(Batch):
    """Batch with a 4-bit cache."""

    def __init__(self, ops, *args, **kw):
        super().__init__(ops, *args, **kw)
        n = self.cache.pool.shape[0]
        self.cache = ops.KvCache.empty(n, self.n_kv, self.hd, self.table, page=self.page, bits=4)
        self.cache.pool.copy_(torch.from_numpy(
            self.rng.integers(0, 256, tuple(self.cache.pool.shape), dtype=np.uint8)))

    def store(self, k, v):
        """Whole contexts appended in one call; what the cache then stands for, per sequence."""
        start = np.concatenate([[0], np.cumsum(self.lens)])
        self.cache.append(k, v, self.length, row_start=ints(start.tolist()))
        kk, vv = oracle.kv4_values(f64(k)), oracle.kv4_values(f64(v))
        return ([kk[a:b] for a, b in zip(start[:-1], start[1:])],
                [vv[a:b] for a, b in zip(start[:-1], start[1:])])

    def fill(self, dtype=F32):
        n = sum(self.lens)
        k, v = (rnd(self.rng, n, self.n_kv, self.hd, dtype=dtype) for _ in "kv")
        k[:, :, 3] *= 5
        return self.store(k, v)


def sub_batch(lens, rows, start):
    bt = Batch.__new__(Batch)
    bt.lens, bt.rows, bt.start = lens, rows, np.asarray(start)
    return bt


def tolerance(want, mag, dots, n, single, out_dtype, top=0.0):
    """top: the largest |v| that each row sees (broadcast to `want`)."""
    e = 64 * 2.0 ** -24 * dots + 2.0 ** -20
    weight = 2.0 ** -11 if single else 2.0 ** -24
    rel = 2 * e + weight + 2 * (64 + n / 16) * 2.0 ** -24
    lost = 3 * n * (2.0 ** -126 + (top >= 2.0 ** 100) * 2.0 ** -94) + \
        (n * 2.0 ** -31 if single else 0.0)
    return mag * rel[..., None] + abs(want) * (torch.finfo(out_dtype).eps / 2) + lost * top + 1e-30


def check_attend(bt, q, out, K, V, scale, seen=None):
    """out [n_rows, heads, hd] of q against the definition, for every row of the batch."""
    qn, on = f64(q), f64(out)
    single = q.dtype == BF16 and out.dtype == BF16
    for b, (n, r) in enumerate(zip(bt.lens, bt.rows)):
        at = slice(bt.start[b], bt.start[b] + r)
        pos = np.arange(n - r, n)
        sees = np.arange(n)[None] <= pos[:, None]
        if seen is not None:
            sees &= seen(b, np.arange(n))[None]
        want, mag, dots = oracle.attend_rows(qn[at], K[b], V[b], sees, scale)
        if not r:
            continue
        top = np.where(sees, np.abs(V[b]).max((1, 2))[None], 0.0).max(1)[:, None, None]
        tol = tolerance(want, mag, dots, n, single, out.dtype, top)
        err = np.abs(on[at] - want)
        assert np.all(err <= tol), (b, float(np.max(err / tol)))


# ------------------------------------------------------------------ append and read
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_stores_the_definitions_bytes(ops, hd, page, dtype):
    lens, rows = [150, 1, 129, 64, 7], [150, 1, 66, 0, 3]
    bt = Batch4(ops, lens, rows, hd=hd, page=page, n_kv=3, seed=page + hd)
    before = bt.cache.pool.clone()
    k, v = (rnd(bt.rng, bt.n_rows, 3, hd, dtype=dtype) for _ in "kv")
    k[0, 0] = 0                                     # nothing: the least scale
    k[1, 0] = 1e-20
    v[1, 0] = 1e-42                                 # (below fp32's normal numbers)
    v[2, 1] *= 1e30
    k[2, 1] = 3.3e38                                # past the largest scale: 6 of it
    k[3, 2, 5], v[4, 0, hd - 1] = float("nan"), -float("inf")
    # every tie, with either sign, and one past; 7 exactly
    ties = torch.tensor([.25, .75, 1.25, 1.75, 2.5, 3.5, 5, 7])
    for x in (k, v):
        x[5, 1, :8], x[5, 1, 8:16], x[5, 1, 16:] = ties, -ties, 0
        x[6, 1, :32], x[6, 1, 32:] = torch.linspace(-7, 7.0625, 32), 0.001
    bt.cache.append(k, v, bt.length, row_start=bt.row_start)
    after = bt.cache.pool.clone()
    touched = np.zeros(tuple(after.shape), bool)
    got = after.cpu().numpy()
    pair, group = np.arange(hd // 2), np.arange(hd // 32)
    for i, (b, p) in enumerate(bt.where()):
        phys, slot = int(bt.table[b, p // page]), p % page
        for which, x in ((0, k), (1, v)):
            code, byte = oracle.kv4_quantise(f64(x[i]))
            at, st = (slot * hd // 2 + pair, slot * (hd // 32) + group) if which == 0 else \
                (slot // 4 * 2 * hd + 4 * pair + slot % 4, slot // 4 * (hd // 8) + 4 * group + slot % 4)
            st = st + page * hd // 2
            for h in range(3):
                touched[phys, which, h, at] = touched[phys, which, h, st] = True
                assert np.array_equal(got[phys, which, h, at], code[h, 0::2] + 16 * code[h, 1::2]), (i, which, h)
                assert np.array_equal(got[phys, which, h, st], byte[h]), (i, which, h)
    assert np.array_equal(got[~touched], before.cpu().numpy()[~touched])
    # read back: the values, rounded once
    for t in (F32, BF16):
        rk, rv = bt.cache.read(bt.length, row_start=bt.row_start, n_rows=bt.n_rows, dtype=t)
        for got_x, x in ((rk, k), (rv, v)):
            want = torch.from_numpy(oracle.kv4_values(f64(x)).astype(np.float32)).to(t)
            assert torch.equal(torch.nan_to_num(got_x.cpu(), nan=7e7), torch.nan_to_num(want, nan=7e7))


@pytest.mark.parametrize("layout,dim,hd", [
    ("half", 128, 128), ("pairs", 128, 128), ("half", 24, 128), ("pairs", 64, 128), ("half", 72, 128),
    ("half", 64, 64), ("pairs", 64, 64), ("half", 24, 64), ("half", 56, 64)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_rotates_keys_and_queries(ops, layout, dim, hd, dtype):
    bt = Batch4(ops, [300, 45, 2], [44, 45, 1], page=32, seed=dim, hd=hd)
    t = ops.rope_table(299, dim, layout=layout, scaling="ramp", factor=4.0, original=100.0)
    k, v = (rnd(bt.rng, bt.n_rows, 2, hd, dtype=dtype) for _ in "kv")
    q = rnd(bt.rng, bt.n_rows, 6, hd, dtype=dtype)
    got_q = bt.cache.append(k, v, bt.length, row_start=bt.row_start, rope=t, q=q)
    pos = np.array([p for _, p in bt.where()])
    c, s = (x.cpu().numpy()[np.minimum(pos, 298)] for x in (t.cos, t.sin))
    turned = oracle.rope_pairs(k.float().cpu().numpy(), c, s, layout)
    want_q = oracle.rope_pairs(q.float().cpu().numpy(), c, s, layout)
    past = pos == 299                                # past the tables: NaN
    turned[past, :, :dim], want_q[past, :, :dim] = np.nan, np.nan
    rk, rv = bt.cache.read(bt.length, row_start=bt.row_start, n_rows=bt.n_rows, dtype=F32)
    for got, want in ((rk, oracle.kv4_values(turned)), (rv, oracle.kv4_values(f64(v)))):
        assert np.array_equal(got.cpu().numpy(), want.astype(np.float32), equal_nan=True)
    want_q = torch.from_numpy(want_q).to(dtype)
    assert torch.equal(torch.nan_to_num(got_q.cpu(), nan=7e7), torch.nan_to_num(want_q, nan=7e7))


def test_single_tokens_append_like_rows(ops):
    bt = Batch4(ops, [1, 16, 17, 100], n_kv=2, hd=128, page=16)
    K, V = bt.fill()
    k, v = (rnd(bt.rng, 4, 4, 128) for _ in "kv")
    bt.cache.append(k[:, 1:3], v[:, 2:], bt.length)   # (strided rows)
    start = np.concatenate([[0], np.cumsum(bt.lens)])
    rk, rv = bt.cache.read(bt.length, row_start=ints(start.tolist()), n_rows=int(start[-1]), dtype=F32)
    for b in range(4):
        K[b][-1], V[b][-1] = oracle.kv4_values(f64(k[b, 1:3])), oracle.kv4_values(f64(v[b, 2:]))
        for got, want in ((rk, K), (rv, V)):
            assert np.array_equal(got[start[b]:start[b + 1]].cpu().numpy(), want[b].astype(np.float32))


def test_rows_of_no_sequence_and_positions_without_pages_are_left(ops):
    bt = Batch4(ops, [40, 30, 100, 3], [40, 30, 2, 5], page=16, pad=(3, 4), extra_pages=0)
    bt.table[0, 1], bt.table[1, 0] = -1, 10 ** 6     # lost pages
    bt.length[2] = 7 * 16 + 1                        # past the 7 entries of the table
    k, v = (rnd(bt.rng, bt.n_rows, 2, 128) for _ in "kv")
    before = bt.cache.pool.clone()
    bt.cache.append(k, v, bt.length, row_start=bt.row_start)
    rk = torch.full((bt.n_rows, 2, 128), 9.0, device="cuda")
    rv = rk.clone()
    bt.cache.read(bt.length, row_start=bt.row_start, k=rk, v=rv)
    changed = (bt.cache.pool != before).flatten(1).any(1).cpu().numpy()
    used = {int(bt.table[0, p]) for p in (0, 2)} | {int(bt.table[1, 1]), int(bt.table[2, 6]),
                                                    int(bt.table[3, 0])}
    assert set(np.flatnonzero(changed)) <= used
    want = {}
    for i, (b, p) in enumerate(bt.where()):
        p += 13 if b == 2 else 0
        lost = (b, p // 16) in ((0, 1), (1, 0)) or p // 16 >= 7
        want[bt.start[0] + i] = None if p < 0 else 0 if lost else 1
    for i in range(bt.n_rows):
        for got, x in ((rk, k), (rv, v)):
            w = want.get(i)
            exp = np.full((2, 128), 9.0) if w is None else oracle.kv4_values(f64(x[i])) * w
            assert np.array_equal(got[i].cpu().numpy(), exp.astype(np.float32)), i


# ------------------------------------------------------------------ attention
@pytest.mark.parametrize("n_kv,G,hd,page", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_single_tokens(ops, n_kv, G, hd, page, dtype):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 700]
    bt = Batch4(ops, lens, n_kv=n_kv, hd=hd, page=page, seed=G)
    K, V = bt.fill()
    q = rnd(bt.rng, len(lens), n_kv * G, hd, dtype=dtype, scale=1.5)
    for hint in (0, 1, 700):
        out = bt.cache.attend(q, bt.length, max_length=hint)
        assert out.dtype == dtype
        check_attend(bt, q, out, K, V, hd ** -0.5)


@pytest.mark.parametrize("n_kv,G,hd,page", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_prompts(ops, n_kv, G, hd, page, dtype):
    """Whole prompts, later chunks, single rows and absent ones in one packed call."""
    lens, rows = [1, 65, 200, 64, 333, 40], [1, 65, 40, 0, 130, 1]
    bt = Batch4(ops, lens, rows, n_kv=n_kv, hd=hd, page=page, seed=G + 50)
    K, V = bt.fill()
    q = rnd(bt.rng, bt.n_rows, n_kv * G, hd, dtype=dtype, scale=1.5)
    for hints in ({}, dict(max_rows=130, max_length=333), dict(max_rows=1, max_length=1)):
        out = bt.cache.attend(q, bt.length, row_start=bt.row_start, **hints)
        check_attend(bt, q, out, K, V, hd ** -0.5)


@pytest.mark.parametrize("n_seqs,rows,length,n_kv,G,hd,entries,page", PLAN_CASES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_kernel(ops, n_seqs, rows, length, n_kv, G, hd, entries, page, dtype):
    """Against float64 on the GPU, all rows; some sequences shorter and with fewer rows, one
    without any."""
    lens = [max(rows, length - 7 * b) for b in range(n_seqs)]
    new = [max(0, rows - b % 4) if b != 1 else 0 for b in range(n_seqs)]
    need = -(-max(lens) // page)
    bt = Batch4(ops, lens, new, n_kv=n_kv, hd=hd, page=page, seed=rows + n_seqs, extra_pages=entries - need)
    K, V = bt.fill(dtype=BF16)
    q = rnd(bt.rng, bt.n_rows, n_kv * G, hd, dtype=dtype, scale=1.5)
    out = bt.cache.attend(q, bt.length, row_start=bt.row_start, max_rows=rows)
    check_on_gpu(bt, q, out, K, V)


def check_on_gpu(bt, q, out, K, V):
    """Against float64 on the GPU, all rows."""
    n_kv, hd, dtype = bt.n_kv, bt.hd, q.dtype
    G = q.shape[1] // n_kv
    for b, (n, r) in enumerate(zip(bt.lens, bt.rows)):
        if not r:
            continue
        at = slice(bt.start[b], bt.start[b] + r)
        k, v = (torch.from_numpy(x).cuda().transpose(0, 1)[:, None].contiguous() for x in (K[b], V[b]))
        qq = q[at].double().view(r, n_kv, G, hd).permute(1, 2, 0, 3).contiguous()
        x = qq @ k.transpose(-1, -2).contiguous() * hd ** -0.5
        late = torch.arange(n, device="cuda")[None] > torch.arange(n - r, n, device="cuda")[:, None]
        p = x.masked_fill(late, float("-inf")).softmax(-1)
        want, mag = p @ v, p @ v.abs()
        dots = (qq.abs() @ k.abs().transpose(-1, -2).contiguous()).amax(-1) * hd ** -0.5
        top = v.abs().amax(-1).cummax(-1).values[..., n - r:, None]
        tol = tolerance(want, mag, dots, n, dtype == BF16, out.dtype, top)
        err = (out[at].double().view(r, n_kv, G, hd).permute(1, 2, 0, 3) - want).abs()
        assert (err <= tol).all(), (b, float((err / tol).max()))


@pytest.mark.parametrize("n_seqs,rows,length,n_kv,G,hd,entries,page", PLAN_CASES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("where", ["early", "late", "here and there"])
def test_values_past_halves(ops, n_seqs, rows, length, n_kv, G, hd, entries, page, dtype, where):
    """Value rows of zeros, of 1e-12 and up to fp32's end, in every kernel: before, after and among
    ordinary ones."""
    lens = [max(rows, length - 7 * b) for b in range(min(n_seqs, 9))]
    lens += [max(rows, length)] * (n_seqs - len(lens))
    need = -(-max(lens) // page)
    bt = Batch4(ops, lens, [rows] * n_seqs, n_kv=n_kv, hd=hd, page=page, seed=rows + n_seqs,
                extra_pages=entries - need)
    n = sum(lens)
    k, v = (rnd(bt.rng, n, n_kv, hd, dtype=F32) for _ in "kv")
    at = np.concatenate([np.arange(x) for x in lens])
    odd = {"early": at < 3, "late": at >= length - rows // 2 - 2,
           "here and there": bt.rng.random(n) < 0.05}[where]
    size = np.where(odd, bt.rng.choice([0.0, 1e-12, 1e7, 1e25, 3e36], n), 1.0)
    if where == "early":
        size[at == 0] = 1e38 / 4
    v *= torch.from_numpy(size.astype(np.float32)).cuda()[:, None, None]
    K, V = bt.store(k, v)
    q = rnd(bt.rng, bt.n_rows, n_kv * G, hd, dtype=dtype, scale=1.5)
    out = bt.cache.attend(q, bt.length, row_start=bt.row_start, max_rows=rows)
    assert out.isfinite().all()
    check_on_gpu(bt, q, out, K, V)


@pytest.mark.parametrize("rows", [None, [3, 16, 700]])
def test_long_contexts(ops, rows):
    lens = [5000, 16, 2111]
    bt = Batch4(ops, lens, rows, n_kv=1, hd=128, page=128)
    K, V = bt.fill()
    for dtype in (BF16, F32):
        q = rnd(bt.rng, bt.n_rows, 4, 128, dtype=dtype, scale=2.0)
        check_attend(bt, q, bt.cache.attend(q, bt.length, row_start=bt.row_start, max_rows=700),
                     K, V, 128 ** -0.5)


@pytest.mark.parametrize("qt,ot", [(BF16, F32), (F32, BF16)])
def test_types_strides_and_scale(ops, qt, ot):
    """Queries inside projection rows, output inside wider rows of the other type, another scale."""
    bt = Batch4(ops, [70, 19], [30, 19], n_kv=2, hd=64, page=32)
    K, V = bt.fill()
    proj = rnd(bt.rng, 49, 12, 64, dtype=qt)
    wide = torch.full((49, 20, 64), 5.0, dtype=ot, device="cuda")
    out = wide.permute(1, 0, 2)[4:12].permute(1, 0, 2)
    bt.cache.attend(proj[:, 2:10], bt.length, row_start=bt.row_start, scale=-0.2, out=out)
    check_attend(bt, proj[:, 2:10], out, K, V, -0.2)
    assert (wide[:, :4] == 5).all() and (wide[:, 12:] == 5).all()


@pytest.mark.parametrize("rows", [None, [150, 9]])
def test_values_and_queries_of_any_magnitude(ops, rows):
    """Value rows from 1e-15 to 1e30 in one context, largest where weights are smallest and
    elsewhere; queries from 1e-20 to 1e10."""
    for seed, (qs, order) in enumerate([(1.0, 1), (1.0, -1), (1e-20, 1), (50.0, 0), (1e10, 0)]):
        bt = Batch4(ops, [200, 90], rows, n_kv=1, hd=128, page=64, seed=seed)
        size = 10.0 ** np.linspace(-15, 30, 290)[::-1 if order < 0 else 1].copy()
        if order == 0:
            bt.rng.shuffle(size)
        k = rnd(bt.rng, 290, 1, 128, dtype=F32)
        v = rnd(bt.rng, 290, 1, 128, dtype=F32) * torch.tensor(size, device="cuda").float()[:, None, None]
        K, V = bt.store(k, v)
        for dtype in (BF16, F32):
            q = rnd(bt.rng, bt.n_rows, 3, 128, dtype=dtype, scale=qs)
            check_attend(bt, q, bt.cache.attend(q, bt.length, row_start=bt.row_start), K, V, 128 ** -0.5)


def test_hints_that_are_wrong(ops):
    """max_rows and max_length below what the batch holds, or far above: the same rows, beyond the
    order of sums; a scale of zero weighs all alike."""
    bt = Batch4(ops, [900, 5, 300], [130, 5, 17], n_kv=2, hd=128, page=16)
    K, V = bt.fill()
    q = rnd(bt.rng, bt.n_rows, 8, 128, dtype=F32)
    for hints in (dict(max_rows=1), dict(max_rows=1, max_length=1), dict(max_length=33),
                  dict(max_rows=2 ** 31 - 1, max_length=2 ** 31 - 1), dict(max_rows=40, max_length=20000)):
        check_attend(bt, q, bt.cache.attend(q, bt.length, row_start=bt.row_start, **hints), K, V,
                     128 ** -0.5)
    for scale in (0.0, -128 ** -0.5):
        check_attend(bt, q, bt.cache.attend(q, bt.length, row_start=bt.row_start, scale=scale), K, V, scale)


def test_rows_that_see_nothing(ops):
    """Length zero, every page absent, more rows than positions: zeros, where garbage (and NaN
    scales) lies in the pages; rows of no sequence are left."""
    bt = Batch4(ops, [50, 33, 40, 4], [2, 33, 1, 6], n_kv=2, hd=128, page=16, pad=(2, 3))
    K, V = bt.fill()
    bt.cache.pool[int(bt.table[2, 2])] = 255         # past position 39 ..
    bt.cache.append(torch.zeros(8, 2, 128, device="cuda"), torch.ones(8, 2, 128, device="cuda"),
                    ints([0, 0, 40]), row_start=ints([0, 0, 0, 8]))
    K[2][32:], V[2][32:] = 0.0, 1.0                  # .. and 32-39 anew
    bt.length[0] = 0
    bt.table[1, :] = -1
    for dtype in (BF16, F32):
        q = rnd(bt.rng, bt.n_rows, 8, 128, dtype=dtype)
        for hints in ({}, dict(max_rows=33, max_length=50), dict(max_rows=33, max_length=4000)):
            out = torch.full_like(q, 7.0)
            bt.cache.attend(q, bt.length, row_start=bt.row_start, out=out, **hints)
            assert (out[:2] == 7).all() and (out[-3:] == 7).all()
            assert not out[2:4].any() and not out[4:37].any() and not out[38:40].any()
            check_attend(sub_batch([40, 4], [1, 4], [37, 40]), q, out, [K[2], K[3]], [V[2], V[3]],
                         128 ** -0.5)


def test_lost_pages_are_not_attended(ops):
    bt = Batch4(ops, [100, 57], [100, 1], n_kv=2, hd=64, page=16)
    K, V = bt.fill()
    bt.table[0, 0], bt.table[0, 3], bt.table[1, 3] = -1, 2 ** 30, -2 ** 31
    gone = {0: (0, 3), 1: (3,)}
    for dtype in (BF16, F32):
        q = rnd(bt.rng, bt.n_rows, 4, 64, dtype=dtype)
        out = bt.cache.attend(q, bt.length, row_start=bt.row_start)
        check_attend(bt, q, out, K, V, 0.125, seen=lambda b, j: ~np.isin(j // 16, gone[b]))
        assert not out[:16].any()                    # rows whose only page is lost


@pytest.mark.parametrize("n_seqs,rows,length,n_kv,G,hd,entries,page", PLAN_CASES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_masked_places_do_not_matter(ops, n_seqs, rows, length, n_kv, G, hd, entries, page, dtype):
    """NaN rows later in a prompt, and NaN or the largest scales past a context's end, do not
    reach earlier rows; a NaN or infinite row reaches exactly the rows that see it: in every
    kernel."""
    lens, new = [length, length], [rows, min(rows, 3)]
    need = -(-length // page)
    bt = Batch4(ops, lens * (n_seqs // 2 + 1), new * (n_seqs // 2 + 1), n_kv=n_kv, hd=hd, page=page,
                extra_pages=entries - need, seed=length)
    bt.fill(dtype=BF16)
    q = rnd(bt.rng, bt.n_rows, n_kv * G, hd, dtype=dtype)

    def attend():
        return bt.cache.attend(q, bt.length, row_start=bt.row_start, max_rows=rows)
    clean = attend()
    # every byte past the last position of the first sequence's last page that holds only such
    phys, used = int(bt.table[0, need - 1]), (length - 1) % page + 1
    four = -(-used // 4) * 4
    if four < page:
        blk = bt.cache.pool[phys]
        blk[0, :, used * hd // 2:page * hd // 2] = 255
        blk[0, :, page * hd // 2 + used * (hd // 32):] = 255
        blk[1, :, four * hd // 2:page * hd // 2] = 255
        blk[1, :, page * hd // 2 + four * (hd // 32):] = 255
        assert torch.equal(attend(), clean)
    # a position among the new rows of the first sequence: a value row with a NaN; then a key row
    at = length - rows // 2 - 1
    for name in "vk":
        one = torch.ones(1, n_kv, hd, device="cuda")
        bad = one.clone()
        bad[0, :, 7] = float("nan") if name == "v" else float("inf")
        bt.cache.append(*((one, bad) if name == "v" else (bad, one)), ints([at + 1]))
        out = attend()
        first = at - (length - rows)
        assert torch.equal(out[:first], clean[:first])
        assert torch.equal(out[rows:], clean[rows:])
        assert out[first:rows].isnan().all()


def test_nan_and_infinite_queries_stay_in_their_rows(ops):
    for n, r in ((70, 10), (400, 300)):
        bt = Batch4(ops, [n], [r], n_kv=1, hd=64, page=16, seed=3)
        bt.fill()
        for t in (BF16, F32):
            q = rnd(bt.rng, r, 4, 64, dtype=t)
            want = bt.cache.attend(q, bt.length, row_start=bt.row_start)
            q[3, 1, 5], q[7, 2, 0] = float("nan"), float("inf")
            out = bt.cache.attend(q, bt.length, row_start=bt.row_start)
            assert out[3, 1].isnan().all() and out[7, 2].isnan().all()
            for i, h in ((3, 1), (7, 2)):
                out[i, h] = want[i, h] = 0
            assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [None, [200]])
def test_scores_past_the_range(ops, dtype, rows):
    """Scores of minus infinity count nothing beside finite ones, one of infinity makes its row
    NaN, and a row whose every score is minus infinity is the quotient of two zeros."""
    bt = Batch4(ops, [700], rows, n_kv=1, hd=64, page=16, seed=9)
    k = rnd(bt.rng, 700, 1, 64, dtype=F32) * 0.01
    k[:, :, 0] = 0
    k[100, 0, 0], k[690, 0, 0] = 2e38, -2e38
    v = rnd(bt.rng, 700, 1, 64, dtype=F32)
    K, V = bt.store(k, v)
    n = bt.n_rows
    q = torch.zeros(n, 2, 64, dtype=dtype, device="cuda")
    q[:, :, 1:] = rnd(bt.rng, n, 2, 63, dtype=dtype)
    q[:, 1, 0] = -20.0                               # position 100: minus infinity
    out = bt.cache.attend(q, bt.length, row_start=bt.row_start)
    late = n - 10 if rows else 0                     # rows that see position 690 (infinity)
    assert out[late:, 1].isnan().all() and not out[:late].isnan().any() and not out[:, 0].isnan().any()
    keep = np.arange(700) != 100
    qq = q.clone()
    qq[:, :, 0] = 0
    check_attend(sub_batch([700], [n], [0]), qq[:, :1].contiguous(), out[:, :1].contiguous(), K, V, 0.125)
    if late:
        want, mag, dots = oracle.attend_rows(f64(qq[:late, 1:]), K[0], V[0],
                                             (np.arange(700)[None] <= (700 - n + np.arange(late))[:, None]) & keep,
                                             0.125)
        tol = tolerance(want, mag, dots, 700, dtype == BF16, dtype, 10.0)
        assert np.all(np.abs(f64(out[:late, 1:]) - want) <= tol)
    k[:, 0, 0] = 2e38
    bt.store(k, v)
    out = bt.cache.attend(q, bt.length, row_start=bt.row_start)
    assert out[:, 1].isnan().all() and not out[:, 0].isnan().any()


def test_equal_scores_however_large(ops):
    """Keys that are all alike weigh alike, also where a score's own rounding exceeds 1."""
    for rows in (None, [130]):
        bt = Batch4(ops, [333], rows, n_kv=1, hd=128, page=32)
        k = rnd(bt.rng, 1, 1, 128, dtype=F32).expand(333, 1, 128).contiguous()
        v = rnd(bt.rng, 333, 1, 128, dtype=F32)
        K, V = bt.store(k, v)
        for t in (BF16, F32):
            for size in (1.0, 1e9, 1e30, -1e30):
                q = rnd(bt.rng, bt.n_rows, 4, 128, dtype=t) * size
                out = bt.cache.attend(q, bt.length, row_start=bt.row_start)
                zero = torch.zeros_like(q)           # the same weights
                check_attend(bt, zero, out, K, V, 1.0)


def test_large_pool_offsets(ops):
    """Pages whose blocks lie past 4 GiB of the pool."""
    n_kv, hd, page = 8, 128, 128
    n_pages = (5 << 30) // (2 * n_kv * page * 68)
    table = ints([[n_pages - 1, 3, n_pages - 2]])
    cache = ops.KvCache.empty(n_pages, n_kv, hd, table, page=page, bits=4)
    rng = np.random.default_rng(4)
    k, v = (rnd(rng, 300, n_kv, hd) for _ in "kv")
    at = dict(row_start=ints([0, 300]))
    cache.append(k, v, ints([300]), **at)
    rk, rv = cache.read(ints([300]), n_rows=300, dtype=F32, **at)
    K, V = oracle.kv4_values(f64(k)), oracle.kv4_values(f64(v))
    assert np.array_equal(rk.cpu().numpy(), K.astype(np.float32))
    assert np.array_equal(rv.cpu().numpy(), V.astype(np.float32))
    q = rnd(rng, 1, 8, hd)
    check_attend(sub_batch([300], [1], [0]), q, cache.attend(q, ints([300])), [K], [V], hd ** -0.5)
    q = rnd(rng, 300, 8, hd)
    check_attend(sub_batch([300], [300], [0]), q, cache.attend(q, ints([300]), **at), [K], [V], hd ** -0.5)


# ------------------------------------------------------------------ together, as they are used
def test_decoding_in_a_graph(ops):
    """Rotation + append + attention of single tokens captured twice and replayed as the
    sequences grow (lengths change in place), against eager calls."""
    rng = np.random.default_rng(8)
    B, H, G, hd, page = 5, 2, 4, 128, 16
    table = ints([[7 * b + i for i in range(7)] for b in range(B)])
    t = ops.rope_table(200, hd)
    caches = [ops.KvCache.empty(7 * B, H, hd, table, page=page, bits=4) for _ in "ab"]
    for c in caches:
        c.pool.zero_()
    lens0 = [1, 15, 16, 40, 63]
    start = np.concatenate([[0], np.cumsum(lens0)])
    pk, pv = (rnd(rng, int(start[-1]), H, hd) for _ in "kv")
    length = ints(lens0)
    for c in caches:
        c.append(pk, pv, length, row_start=ints(start.tolist()), rope=t)
    q, k, v = (rnd(rng, B, n, hd) for n in (H * G, H, H))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def step(c):
        return c.attend(c.append(k, v, length, rope=t, q=q), length)

    with torch.cuda.stream(s):
        for c in caches:
            step(c)
    s.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(step(caches[1]))
        graphs.append(g)
    for i in range(6):
        length += 1
        for x in (q, k, v):
            x.copy_(rnd(rng, *x.shape))
        eager = step(caches[0])
        torch.cuda.synchronize()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[i % 2], eager), i
    assert torch.equal(caches[0].pool, caches[1].pool)


def test_prompt_then_tokens_is_one_long_prompt(ops):
    """A prompt in chunks and then token by token leaves the cache that one call does, and gives
    the rows."""
    rng = np.random.default_rng(9)
    n, H, G, hd, page = 150, 2, 4, 64, 32
    table = ints([[4, 0, 3, 1, 2]])
    a, b = (ops.KvCache.empty(5, H, hd, table, page=page, bits=4) for _ in "ab")
    for c in (a, b):
        c.pool.zero_()
    t = ops.rope_table(n, hd, layout="pairs")
    q, k, v = (rnd(rng, n, x, hd, dtype=F32) for x in (H * G, H, H))
    full = a.attend(a.append(k, v, ints([n]), row_start=ints([0, n]), rope=t, q=q), ints([n]),
                    row_start=ints([0, n]))
    parts = []
    for lo, hi in [(0, 70), (70, 71), (71, 143)] + [(i, i + 1) for i in range(143, n)]:
        at = dict(row_start=ints([0, hi - lo]))
        qq = b.append(k[lo:hi], v[lo:hi], ints([hi]), rope=t, q=q[lo:hi], **at)
        parts.append(b.attend(qq, ints([hi]), **at))
    assert torch.equal(a.pool, b.pool)
    # both within the bound of check_attend; rows of unit scale: 2^-17 covers twice that
    assert (torch.cat(parts) - full).abs().max() <= 2.0 ** -17 * 4


def test_workspace_and_two_streams(ops):
    """Calls at once on two streams, each with a workspace of its own; out may be q."""
    bt = Batch4(ops, [3000] * 2, n_kv=1, hd=64, page=64)
    bt.fill()
    q = rnd(bt.rng, 2, 4, 64)
    need = bt.cache.attend_workspace(2, 4, 2)
    assert need > 0
    want = bt.cache.attend(q, bt.length)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in "ab"]
    spaces = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in "ab"]
    outs = [bt.cache.attend(q, bt.length, workspace=w, stream=s)
            for _ in range(10) for s, w in zip(streams, spaces)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    with pytest.raises(Exception, match="WICI_E_ARG"):
        bt.cache.attend(q, bt.length, workspace=spaces[0][:-1])
    assert bt.cache.attend(q, bt.length, out=q) is q and torch.equal(q, want)


def test_python_refusals(ops):
    bt = Batch4(ops, [5, 6], n_kv=2, hd=64, page=16)
    k = torch.zeros(2, 2, 64, device="cuda")
    for call in (lambda: bt.cache.append(k.half(), k, bt.length),
                 lambda: bt.cache.append(k, k, bt.length, rope=ops.rope_table(8, 128)),
                 lambda: bt.cache.attend(k[:, :, :32], bt.length),
                 lambda: bt.cache.append(k.requires_grad_(), k, bt.length),
                 lambda: ops.KvCache(bt.cache.pool, bt.table, page=16, head_dim=64),
                 lambda: ops.KvCache(bt.cache.pool, bt.table, page=16, head_dim=64, bits=5),
                 lambda: ops.KvCache(bt.cache.pool, bt.table, page=32, head_dim=64, bits=4),
                 lambda: ops.KvCache.empty(2, 2, 96, bt.table, page=16, bits=4)):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            call()
