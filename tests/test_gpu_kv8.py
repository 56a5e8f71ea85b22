"""Rotary positions, the 8-bit key-value cache and attention over it, against their
definitions in float64 (oracle/kv8.py).

Tolerances.  Codes, steps and fp32 rotations have one right answer and are compared for
equality (a bf16 result with the rounding of that answer).  Attention: with S the largest
sum |q_d k_d| scale of a row and A the output with |v| in place of v, a score is off by at
most e = (48 2^-24 + [fp32 rows: 2^-22]) S + 2^-20 (a sum of 128 products in fp32, two fp16
terms of the query, the exponential's argument and result), which moves a weight and the sum
by e each; a weight is off by at most 2^-11 (one fp16 term, bf16 rows) or 2^-22 (two) of itself;
the sums over n positions add at most (64 + n / 16) roundings of 2^-24 A; and the result is
rounded once, by eps / 2 of itself."""

from __future__ import annotations

import numpy as np
import pytest

import oracle

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_24204_amd import ops
    return ops


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def rnd(rng, *shape, dtype=BF16, scale=1.0):
    return (torch.from_numpy(rng.standard_normal(shape).astype(np.float32)) * scale).to(dtype).cuda()


def f64(x):
    return x.detach().float().cpu().numpy().astype(np.float64)


class Batch:
    """Sequences of `lens` positions, the last `rows` of each new (None: one each, without
    row_start), in shuffled pages of a pool of random bytes."""

    def __init__(self, ops, lens, rows=None, *, n_kv=2, hd=128, page=16, seed=0, extra_pages=2, pad=(0, 0)):
        rng = np.random.default_rng(seed)
        self.rng, self.lens, self.hd, self.n_kv, self.page = rng, list(lens), hd, n_kv, page
        self.rows = [1] * len(lens) if rows is None else list(rows)
        need = [-(-max(n, 1) // page) for n in lens]
        order = rng.permutation(sum(need) + 1)
        table = rng.integers(-2 ** 31, 2 ** 31, (len(lens), max(need) + extra_pages))
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        self.table = ints(table.tolist())
        self.cache = ops.KvCache.empty(len(order), n_kv, hd, self.table, page=page)
        self.cache.pool.copy_(torch.from_numpy(
            rng.integers(0, 256, tuple(self.cache.pool.shape), dtype=np.uint8)))
        self.length = ints(self.lens)
        start = np.concatenate([[0], np.cumsum(self.rows)]) + pad[0]
        self.row_start = None if rows is None else ints(start.tolist())
        self.n_rows = int(start[-1]) + pad[1]
        self.start = start

    def where(self):
        """(sequence, position) of each row."""
        return [(b, n - r + i) for b, (n, r) in enumerate(zip(self.lens, self.rows)) for i in range(r)]

    def fill(self, scale=1.0, dtype=F32):
        """Whole contexts appended in one call; returns what the cache then stands for, per
        sequence [n, n_kv, hd]."""
        n = sum(self.lens)
        k, v = (rnd(self.rng, n, self.n_kv, self.hd, dtype=dtype, scale=scale) for _ in "kv")
        k[:, :, 3] *= 5
        start = np.concatenate([[0], np.cumsum(self.lens)])
        self.cache.append(k, v, self.length, row_start=ints(start.tolist()))
        kk, vv = oracle.kv8_values(f64(k)), oracle.kv8_values(f64(v))
        return ([kk[a:b] for a, b in zip(start[:-1], start[1:])],
                [vv[a:b] for a, b in zip(start[:-1], start[1:])])

    def blocks(self, b, p):
        """The bytes of logical page p of sequence b: [2, n_kv, block]."""
        return self.cache.pool[int(self.table[b, p])].cpu().numpy()


def check_attend(bt, q, out, K, V, scale, seen=None, far=False):
    """out [n_rows, heads, hd] of q against the definition, for every row of the batch.

    far: with weights 2^-20 and more below the largest W of a row, which fp16 holds only to the
    half of its least step, 2^-25, where W is 2^6 or more: to 2^-31 W.  W is p_j t_j of some
    position j, of which a code is 127 in some dimension, so that 127 W <= max_d A_d; codes
    are at most 127, so n such errors add at most n 2^-31 max_d A_d to a dimension."""
    qn, on = f64(q), f64(out)
    for b, (n, r) in enumerate(zip(bt.lens, bt.rows)):
        at = slice(bt.start[b], bt.start[b] + r)
        pos = np.arange(n - r, n)
        sees = np.arange(n)[None] <= pos[:, None]
        if seen is not None:
            sees &= seen(b, np.arange(n))[None]
        want, mag, dots = oracle.attend_rows(qn[at], K[b], V[b], sees, scale)
        single = q.dtype == BF16 and out.dtype == BF16
        e = (48 * 2.0 ** -24 + (0 if single else 2.0 ** -22)) * dots + 2.0 ** -20
        rel = 2 * e + (2.0 ** -11 if single else 2.0 ** -22) + (64 + n / 16) * 2.0 ** -24
        tol = mag * rel[..., None] + np.abs(want) * torch.finfo(out.dtype).eps / 2 + 1e-30
        if far:
            tol += n * 2.0 ** -31 * mag.max(-1, keepdims=True)
        err = np.abs(on[at] - want)
        assert np.all(err <= tol), (b, float(np.max(err / tol)))


# ------------------------------------------------------------------ rotary positions
@pytest.mark.parametrize("scaling,kw", [
    ("plain", {}), ("linear", dict(factor=4.0)), ("base", dict(factor=8.0)),
    ("bands", dict(factor=8.0, original=8192.0)),
    ("bands", dict(factor=2.0, original=500.0, low=0.5, high=9.0)),
    ("ramp", dict(factor=16.0, original=4096.0)),
    ("ramp", dict(factor=4.0, original=300.0, low=2.0, high=16.0)), ("ramp", dict(factor=1.0, original=9.0))])
@pytest.mark.parametrize("dim,base", [(8, 100.0), (64, 10000.0), (128, 500000.0)])
def test_rope_tables(ops, scaling, kw, dim, base):
    n = 131072 if dim == 64 else 777
    t = ops.rope_table(n, dim, base=base, scaling=scaling, **kw)
    f, mult = oracle.rope_steps(dim, base, scaling, **kw)
    ang = np.arange(n)[:, None] * f
    for got, want in ((t.cos, mult * np.cos(ang)), (t.sin, mult * np.sin(ang))):
        # one rounding (half a step of a value below 2), and the angle's own in 64 bits
        assert got.shape == want.shape
        assert np.max(np.abs(f64(got) - want)) <= 2.0 ** -24 + n * 2.0 ** -50


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("hd,dim", [(64, 64), (64, 8), (128, 128), (128, 64), (128, 40)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rope_rows(ops, layout, hd, dim, dtype):
    rng = np.random.default_rng(dim)
    n, heads = 37, 3
    t = ops.rope_table(5000, dim, layout=layout, base=10000.0)
    pos = rng.integers(0, 5000, n)
    pos[:3] = 0, 4999, 17
    x = rnd(rng, n, heads, hd, dtype=dtype)
    x[5, 1, 0], x[6, 2, dim - 1] = float("inf"), float("nan")
    got = ops.rope(x, ints(pos.tolist()), t)
    xs = x.float().cpu().numpy()
    want = oracle.rope_pairs(xs, t.cos.cpu().numpy()[pos], t.sin.cpu().numpy()[pos], layout)
    assert torch.equal(torch.nan_to_num(got.cpu(), nan=7e7),
                       torch.nan_to_num(torch.from_numpy(want).to(dtype), nan=7e7))
    assert torch.equal(got[..., dim:], x[..., dim:])
    # in place, and on strided rows of a wider array
    wide = torch.zeros(n, heads + 2, hd, dtype=dtype, device="cuda")
    part = wide[:, 1:heads + 1]
    part.copy_(x)
    assert ops.rope(part, ints(pos.tolist()), t, out=part) is part
    assert torch.equal(torch.nan_to_num(part, nan=7e7), torch.nan_to_num(got, nan=7e7))
    assert not wide[:, 0].any() and not wide[:, -1].any()


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("hd,dim", [(128, 16), (128, 48), (128, 112), (128, 120), (64, 16), (64, 48), (64, 56)])
@pytest.mark.parametrize("xt,ot", [(BF16, BF16), (BF16, F32), (F32, BF16)])
def test_rope_rows_of_other_widths_and_types(ops, layout, hd, dim, xt, ot):
    rng = np.random.default_rng(dim + 1)
    n, heads = 301, 5
    t = ops.rope_table(400, dim, layout=layout, base=10000.0)
    pos = rng.integers(0, 400, n)
    x = rnd(rng, n, heads, hd, dtype=xt)
    out = torch.full((n, heads, hd), 7.0, dtype=ot, device="cuda")
    ops.rope(x, ints(pos.tolist()), t, out=out)
    want = oracle.rope_pairs(x.float().cpu().numpy(), t.cos.cpu().numpy()[pos], t.sin.cpu().numpy()[pos],
                             layout)
    assert torch.equal(out.cpu(), torch.from_numpy(want).to(ot))


def test_rope_rows_outside_the_table(ops):
    t = ops.rope_table(10, 64)
    x = rnd(np.random.default_rng(1), 5, 2, 128)
    out = torch.full_like(x, 3.0)
    ops.rope(x, ints([-1, 9, 10, 2 ** 31 - 1, -2 ** 31]), t, out=out)
    assert (out[0] == 3).all() and (out[4] == 3).all() and out[1].isfinite().all()
    for i in (2, 3):
        assert out[i, :, :64].isnan().all() and torch.equal(out[i, :, 64:], x[i, :, 64:])


# ------------------------------------------------------------------ append and read
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_stores_the_definitions_bytes(ops, hd, page, dtype):
    lens, rows = [150, 1, 129, 64, 7], [150, 1, 66, 0, 3]
    bt = Batch(ops, lens, rows, hd=hd, page=page, n_kv=3, seed=page + hd)
    before = bt.cache.pool.clone()
    k, v = (rnd(bt.rng, bt.n_rows, 3, hd, dtype=dtype) for _ in "kv")
    k[0, 0] = 0                                     # nothing: the least step
    k[1, 0] = 1e-20
    v[2, 1] *= 1e30
    k[3, 2, 5], v[4, 0, hd - 1] = float("nan"), -float("inf")
    k[5, 1, :8] = torch.tensor([254., 1, 3, -1, -3, 5, 0, 2])   # ties
    k[5, 1, 8:] = 0
    bt.cache.append(k, v, bt.length, row_start=bt.row_start)
    after = bt.cache.pool.clone()
    touched = np.zeros(tuple(after.shape), bool)
    got = after.cpu().numpy()
    for i, (b, p) in enumerate(bt.where()):
        phys, slot = int(bt.table[b, p // page]), p % page
        for which, x in ((0, k), (1, v)):
            n, step = oracle.kv8_quantise(f64(x[i]))
            for h in range(3):
                d = np.arange(hd)
                at = slot * hd + d if which == 0 else slot // 4 * 4 * hd + 4 * d + slot % 4
                st = page * hd + 4 * slot + np.arange(4)
                touched[phys, which, h, at] = touched[phys, which, h, st] = True
                assert np.array_equal(got[phys, which, h, at], n[h] + 128), (i, which, h)
                assert np.array_equal(got[phys, which, h, st].view("<f4")[0], step[h], equal_nan=True)
    assert np.array_equal(got[~touched], before.cpu().numpy()[~touched])
    # read back: the values, rounded once
    for t in (F32, BF16):
        rk, rv = bt.cache.read(bt.length, row_start=bt.row_start, n_rows=bt.n_rows, dtype=t)
        for got_x, x in ((rk, k), (rv, v)):
            want = torch.from_numpy(oracle.kv8_values(f64(x)).astype(np.float32)).to(t)
            assert torch.equal(torch.nan_to_num(got_x.cpu(), nan=7e7), torch.nan_to_num(want, nan=7e7))


@pytest.mark.parametrize("layout,dim", [("half", 128), ("pairs", 128), ("half", 24), ("pairs", 64)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_rotates_keys_and_queries(ops, layout, dim, dtype):
    bt = Batch(ops, [300, 45, 2], [44, 45, 1], page=32, seed=dim)
    t = ops.rope_table(299, dim, layout=layout, scaling="ramp", factor=4.0, original=100.0)
    k, v = (rnd(bt.rng, bt.n_rows, 2, 128, dtype=dtype) for _ in "kv")
    q = rnd(bt.rng, bt.n_rows, 6, 128, dtype=dtype)
    got_q = bt.cache.append(k, v, bt.length, row_start=bt.row_start, rope=t, q=q)
    pos = np.array([p for _, p in bt.where()])
    c, s = (x.cpu().numpy()[np.minimum(pos, 298)] for x in (t.cos, t.sin))
    turned = oracle.rope_pairs(k.float().cpu().numpy(), c, s, layout)
    want_q = oracle.rope_pairs(q.float().cpu().numpy(), c, s, layout)
    past = pos == 299                                # past the tables: NaN
    turned[past, :, :dim], want_q[past, :, :dim] = np.nan, np.nan
    assert past.sum() == 1
    rk, rv = bt.cache.read(bt.length, row_start=bt.row_start, n_rows=bt.n_rows, dtype=F32)
    for got, want in ((got_q, torch.from_numpy(want_q).to(dtype)),
                      (rk, torch.from_numpy(oracle.kv8_values(turned).astype(np.float32))),
                      (rv, torch.from_numpy(oracle.kv8_values(f64(v)).astype(np.float32)))):
        assert torch.equal(torch.nan_to_num(got.cpu(), nan=7e7), torch.nan_to_num(want, nan=7e7))
    # the same in place, and without the queries
    assert bt.cache.append(k, v, bt.length, row_start=bt.row_start, rope=t, q=q, q_out=q) is q
    assert torch.equal(torch.nan_to_num(q, nan=7e7), torch.nan_to_num(got_q, nan=7e7))
    assert bt.cache.append(k, v, bt.length, row_start=bt.row_start, rope=t) is None
    assert torch.equal(torch.nan_to_num(bt.cache.read(bt.length, row_start=bt.row_start,
                                                      n_rows=bt.n_rows, dtype=F32)[0], nan=7e7),
                       torch.nan_to_num(rk, nan=7e7))


def test_single_tokens_append_like_rows(ops):
    """One row a sequence, without row_start, at each place in a group of four positions, onto
    what the positions before left."""
    bt = Batch(ops, [1, 2, 3, 4, 5, 64, 65], hd=64, page=16, n_kv=4)
    K, V = bt.fill()
    k, v = (rnd(bt.rng, 7, 4, 64) for _ in "kv")
    bt.cache.append(k, v, bt.length)
    start = np.concatenate([[0], np.cumsum(bt.lens)])
    rk, rv = bt.cache.read(bt.length, row_start=ints(start.tolist()), n_rows=int(start[-1]), dtype=F32)
    for b, n in enumerate(bt.lens):
        K[b][-1], V[b][-1] = oracle.kv8_values(f64(k[b])), oracle.kv8_values(f64(v[b]))
        for got, want in ((rk, K), (rv, V)):
            assert np.array_equal(got[start[b]:start[b + 1]].cpu().numpy(), want[b].astype(np.float32))


def test_rows_of_no_sequence_and_positions_without_pages_are_left(ops):
    """Padding before the first and after the last sequence, pages that are not there, positions
    past the table, more rows than positions: nothing is written, reads give zeros for
    absent pages and leave the other rows, and nothing else changes."""
    bt = Batch(ops, [40, 30, 100, 3], [40, 30, 2, 5], page=16, pad=(3, 4), extra_pages=0)
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
    assert sum(w is None for w in want.values()) == 2 and 0 in want.values()
    for i in range(bt.n_rows):
        for got, x in ((rk, k), (rv, v)):
            w = want.get(i)
            exp = np.full((2, 128), 9.0) if w is None else oracle.kv8_values(f64(x[i])) * w
            assert np.array_equal(got[i].cpu().numpy(), exp.astype(np.float32)), i


# ------------------------------------------------------------------ attention
SHAPES = [  # n_kv, query heads a KV head, head_dim, page
    (2, 4, 128, 64), (1, 8, 64, 16), (3, 1, 128, 16), (2, 5, 64, 128), (1, 20, 128, 32), (8, 2, 64, 32)]


@pytest.mark.parametrize("n_kv,G,hd,page", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_single_tokens(ops, n_kv, G, hd, page, dtype):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 700]
    bt = Batch(ops, lens, n_kv=n_kv, hd=hd, page=page, seed=G)
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
    bt = Batch(ops, lens, rows, n_kv=n_kv, hd=hd, page=page, seed=G + 50)
    K, V = bt.fill()
    q = rnd(bt.rng, bt.n_rows, n_kv * G, hd, dtype=dtype, scale=1.5)
    for hints in ({}, dict(max_rows=130, max_length=333), dict(max_rows=1, max_length=1)):
        out = bt.cache.attend(q, bt.length, row_start=bt.row_start, **hints)
        check_attend(bt, q, out, K, V, hd ** -0.5)


# Calls that between them meet every kernel of the attention (which one a call takes is
# read off the launch rules in test_kv8_host.py): sequences, new rows and positions of each, KV
# heads, query heads a KV head, head size, page-table entries, page.
PLAN_CASES = [
    (1, 37, 90, 2, 2, 128, 8, 16), (1, 37, 90, 2, 2, 64, 8, 16),              # split, one
    (2, 5, 700, 2, 2, 128, 50, 16), (2, 5, 700, 2, 2, 64, 50, 16),            # split, several
    (26, 8, 40, 8, 16, 128, 4, 16), (26, 8, 40, 8, 16, 64, 4, 16),            # 64 rows
    (1, 390, 400, 25, 4, 128, 26, 16), (1, 390, 400, 25, 4, 64, 26, 16),
    (52, 8, 70, 8, 16, 128, 6, 16), (52, 8, 70, 8, 16, 64, 6, 16),            # 128 rows, one
    (2, 700, 730, 8, 5, 128, 6, 128), (2, 700, 730, 8, 5, 64, 6, 128),
    (1, 130, 200, 4, 5, 128, 2100, 128), (1, 130, 200, 4, 5, 64, 2100, 128),  # 128 rows, several
]


@pytest.mark.parametrize("n_seqs,rows,length,n_kv,G,hd,entries,page", PLAN_CASES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_kernel(ops, n_seqs, rows, length, n_kv, G, hd, entries, page, dtype):
    """Against float64 on the GPU, all rows; some sequences shorter and with fewer rows, one
    without any."""
    lens = [max(rows, length - 7 * b) for b in range(n_seqs)]
    new = [max(0, rows - b % 4) if b != 1 else 0 for b in range(n_seqs)]
    need = -(-max(lens) // page)
    bt = Batch(ops, lens, new, n_kv=n_kv, hd=hd, page=page, seed=rows + n_seqs, extra_pages=entries - need)
    K, V = bt.fill(dtype=BF16)
    q = rnd(bt.rng, bt.n_rows, n_kv * G, hd, dtype=dtype, scale=1.5)
    out = bt.cache.attend(q, bt.length, row_start=bt.row_start, max_rows=rows)
    single = dtype == BF16
    for b, (n, r) in enumerate(zip(lens, new)):
        if not r:
            continue
        at = slice(bt.start[b], bt.start[b] + r)
        k, v = (torch.from_numpy(x).cuda().transpose(0, 1)[:, None].contiguous() for x in (K[b], V[b]))
        qq = q[at].double().view(r, n_kv, G, hd).permute(1, 2, 0, 3).contiguous()
        x = qq @ k.transpose(-1, -2).contiguous() * hd ** -0.5
        late = torch.arange(n, device="cuda")[None] > torch.arange(n - r, n, device="cuda")[:, None]
        p = x.masked_fill(late, float("-inf")).softmax(-1)
        want, mag = p @ v, p @ v.abs()
        dots = (qq.abs() @ k.abs().transpose(-1, -2).contiguous()).amax(-1, keepdim=True) * hd ** -0.5
        e = (48 * 2.0 ** -24 + (0 if single else 2.0 ** -22)) * dots + 2.0 ** -20
        rel = 2 * e + (2.0 ** -11 if single else 2.0 ** -22) + (64 + n / 16) * 2.0 ** -24
        tol = mag * rel + want.abs() * torch.finfo(dtype).eps / 2 + 1e-30
        err = (out[at].double().view(r, n_kv, G, hd).permute(1, 2, 0, 3) - want).abs()
        assert (err <= tol).all(), (b, float((err / tol).max()))


def test_many_fp32_rows(ops):
    """20000 rows and heads whose weights are spread over many positions: the two terms of each
    weight belong together in every one of them (an error of one fp16 step in one weight of
    some hundred shows)."""
    n, H, G, hd = 320, 8, 8, 128
    bt = Batch(ops, [n], [n], n_kv=H, hd=hd, page=64, seed=77)
    K, V = bt.fill()
    q = rnd(bt.rng, n, H * G, hd, dtype=F32)
    out = bt.cache.attend(q, bt.length, row_start=bt.row_start).double()
    k, v = (torch.from_numpy(x[0]).cuda().transpose(0, 1) for x in (K, V))        # [H, n, hd]
    x = (q.double().view(n, H, G, hd).permute(1, 2, 0, 3) @ k[:, None].transpose(-1, -2)) * hd ** -0.5
    x = x.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), float("-inf"))
    p = x.softmax(-1)
    want, mag = p @ v[:, None], p @ v[:, None].abs()
    dots = (q.double().abs().view(n, H, G, hd).permute(1, 2, 0, 3) @ k[:, None].abs().transpose(-1, -2)
            ).amax(-1, keepdim=True) * hd ** -0.5
    e = (48 * 2.0 ** -24 + 2.0 ** -22) * dots + 2.0 ** -20
    tol = mag * (2 * e + 2.0 ** -22 + (64 + n / 16) * 2.0 ** -24) + want.abs() * 2.0 ** -24
    assert want.isfinite().all() and tol.isfinite().all() and out.isfinite().all()
    err = (out.view(n, H, G, hd).permute(1, 2, 0, 3) - want).abs()
    assert (err <= tol).all(), float((err / (tol + 1e-30)).max())


@pytest.mark.parametrize("rows", [None, [3, 16, 700]])
def test_long_contexts(ops, rows):
    lens = [5000, 16, 2111] if rows is None else [5000, 16, 2111]
    bt = Batch(ops, lens, rows, n_kv=1, hd=128, page=128)
    K, V = bt.fill()
    for dtype in (BF16, F32):
        q = rnd(bt.rng, bt.n_rows, 4, 128, dtype=dtype, scale=2.0)
        check_attend(bt, q, bt.cache.attend(q, bt.length, row_start=bt.row_start, max_rows=700),
                     K, V, 128 ** -0.5)


@pytest.mark.parametrize("qt,ot", [(BF16, F32), (F32, BF16)])
def test_types_strides_and_scale(ops, qt, ot):
    """Queries inside projection rows, output inside wider rows of the other type, another scale."""
    bt = Batch(ops, [70, 19], [30, 19], n_kv=2, hd=64, page=32)
    K, V = bt.fill()
    proj = rnd(bt.rng, 49, 12, 64, dtype=qt)
    wide = torch.full((49, 20, 64), 5.0, dtype=ot, device="cuda")
    out = wide.permute(1, 0, 2)[4:12].permute(1, 0, 2)
    bt.cache.attend(proj[:, 2:10], bt.length, row_start=bt.row_start, scale=-0.2, out=out)
    check_attend(bt, proj[:, 2:10], out, K, V, -0.2)
    assert (wide[:, :4] == 5).all() and (wide[:, 12:] == 5).all()


def test_values_of_any_magnitude(ops):
    """Value rows from 1e-15 to 1e30 in one context (their scales span 2^150), with the
    largest where the weights are smallest and elsewhere; queries from 1e-20 to 1e10."""
    for seed, (qs, order) in enumerate([(1.0, 1), (1.0, -1), (1e-20, 1), (50.0, 0), (1e10, 0)]):
        bt = Batch(ops, [200, 90], n_kv=1, hd=128, page=64, seed=seed)
        n = 290
        size = 10.0 ** np.linspace(-15, 30, n)[::-1 if order < 0 else 1].copy()
        if order == 0:
            bt.rng.shuffle(size)
        k = rnd(bt.rng, n, 1, 128, dtype=F32)
        v = rnd(bt.rng, n, 1, 128, dtype=F32) * torch.tensor(size, device="cuda").float()[:, None, None]
        bt.cache.append(k, v, bt.length, row_start=ints([0, 200, 290]))
        K, V = ([oracle.kv8_values(f64(x))[a:b] for a, b in ((0, 200), (200, 290))] for x in (k, v))
        for dtype in (BF16, F32):
            q = rnd(bt.rng, 2, 3, 128, dtype=dtype, scale=qs)
            check_attend(bt, q, bt.cache.attend(q, bt.length), K, V, 128 ** -0.5)


def test_queries_of_any_magnitude_in_one_tile(ops):
    """Rows and heads from 1e-9 to 1e9 (and one of 1e38 on keys of 1e-38) beside each other, in
    every order, for single tokens and for prompts: each row's precision is its own."""
    for rows in (None, [40, 9]):
        bt = Batch(ops, [150, 90], rows, n_kv=2, hd=64, page=32, seed=5)
        K, V = bt.fill()
        for dtype in (BF16, F32):
            q = rnd(bt.rng, bt.n_rows, 6, 64, dtype=F32)
            size = 10.0 ** bt.rng.uniform(-9, 9, (bt.n_rows, 6, 1))
            size[bt.rng.random(size.shape) < 0.4] = 1.0
            q = (q * torch.from_numpy(size).float().cuda()).to(dtype)
            check_attend(bt, q, bt.cache.attend(q, bt.length, row_start=bt.row_start), K, V, 0.125,
                         far=True)
    bt = Batch(ops, [60], [20], n_kv=1, hd=128, page=16, seed=6)
    k, v = (rnd(bt.rng, 60, 1, 128, dtype=F32) for _ in "kv")
    k *= 1e-18
    bt.cache.append(k, v, bt.length, row_start=ints([0, 60]))
    K, V = ([oracle.kv8_values(f64(x))] for x in (k, v))
    for dtype in (BF16, F32):
        q = rnd(bt.rng, 20, 4, 128, dtype=F32).clamp(-3, 3)
        q[::3] *= 1e38
        q[1::3] *= 1e18
        q = q.to(dtype)
        check_attend(bt, q, bt.cache.attend(q, bt.length, row_start=bt.row_start, scale=1e-20), K, V,
                     1e-20, far=True)


def test_hints_that_are_wrong(ops):
    """max_rows and max_length below what the batch holds (a plan captured for a small batch), or
    far above: the same rows, beyond the order of sums; a scale of zero weighs all alike."""
    bt = Batch(ops, [900, 5, 300], [130, 5, 17], n_kv=2, hd=128, page=16)
    K, V = bt.fill()
    q = rnd(bt.rng, bt.n_rows, 8, 128, dtype=F32)
    for hints in (dict(max_rows=1), dict(max_rows=1, max_length=1), dict(max_length=33),
                  dict(max_rows=2 ** 31 - 1, max_length=2 ** 31 - 1), dict(max_rows=40, max_length=20000)):
        check_attend(bt, q, bt.cache.attend(q, bt.length, row_start=bt.row_start, **hints), K, V,
                     128 ** -0.5)
    for scale in (0.0, -128 ** -0.5):
        check_attend(bt, q, bt.cache.attend(q, bt.length, row_start=bt.row_start, scale=scale), K, V, scale)


def test_rows_that_see_nothing(ops):
    """Length zero, every page absent, more rows than positions: zeros, where garbage lies in
    the pages; and rows of no sequence are left."""
    bt = Batch(ops, [50, 33, 40, 4], [2, 33, 1, 6], n_kv=2, hd=128, page=16, pad=(2, 3))
    K, V = bt.fill()
    bt.cache.pool.view(torch.float32)[int(bt.table[2, 2])] = float("nan")   # past position 39 ..
    bt.cache.append(torch.zeros(8, 2, 128, device="cuda"), torch.ones(8, 2, 128, device="cuda"),
                    ints([0, 0, 40]), row_start=ints([0, 0, 0, 8]))
    K[2][32:], V[2][32:] = 0.0, 1.0                                          # .. and 32-39 anew
    V[2][32:] = oracle.kv8_values(np.ones((1, 2, 128)))
    bt.length[0] = 0
    bt.table[1, :] = -1
    for dtype in (BF16, F32):
        q = rnd(bt.rng, bt.n_rows, 8, 128, dtype=dtype)
        for hints in ({}, dict(max_rows=33, max_length=50), dict(max_rows=33, max_length=4000)):
            out = torch.full_like(q, 7.0)
            bt.cache.attend(q, bt.length, row_start=bt.row_start, out=out, **hints)
            assert (out[:2] == 7).all() and (out[-3:] == 7).all()
            assert not out[2:4].any() and not out[4:37].any() and not out[38:40].any()
            sub = Batch.__new__(Batch)
            sub.lens, sub.rows, sub.start = [40, 4], [1, 4], np.array([37, 40])
            check_attend(sub, q, out, [K[2], K[3]], [V[2], V[3]], 128 ** -0.5)


def test_lost_pages_are_not_attended(ops):
    bt = Batch(ops, [100, 57], [100, 1], n_kv=2, hd=64, page=16)
    K, V = bt.fill()
    bt.table[0, 0], bt.table[0, 3], bt.table[1, 3] = -1, 2 ** 30, -2 ** 31
    gone = {0: (0, 3), 1: (3,)}
    for dtype in (BF16, F32):
        q = rnd(bt.rng, bt.n_rows, 4, 64, dtype=dtype)
        out = bt.cache.attend(q, bt.length, row_start=bt.row_start)
        check_attend(bt, q, out, K, V, 0.125, seen=lambda b, j: ~np.isin(j // 16, gone[b]))
        assert not out[:16].any()                    # rows whose only page is lost


def test_masked_places_do_not_matter(ops):
    """NaN rows later in a prompt, and NaN or the largest scales past a context's end, do not
    reach earlier rows; a NaN or infinite row reaches exactly the rows that see it."""
    bt = Batch(ops, [64, 90], [64, 20], n_kv=1, hd=128, page=32)
    K, V = bt.fill()
    q = {t: rnd(bt.rng, bt.n_rows, 4, 128, dtype=t) for t in (BF16, F32)}
    clean = {t: bt.cache.attend(q[t], bt.length, row_start=bt.row_start) for t in q}
    # the slots past position 89 of the last page, in every scale's place
    blk = bt.cache.pool.view(torch.float32)[int(bt.table[1, 2])]
    blk[:, :, 32 * 32 + 26:] = torch.tensor([float("nan"), float("inf"), 3e38] * 2, device="cuda")
    for t in q:
        assert torch.equal(bt.cache.attend(q[t], bt.length, row_start=bt.row_start), clean[t])
    # position 40 of the first sequence: a value row with a NaN; then a key row
    for name in "vk":
        bad = torch.ones(1, 1, 128, device="cuda")
        bad[0, 0, 7] = float("nan") if name == "v" else float("inf")
        one = torch.ones_like(bad)
        bt.cache.append(*((one, bad) if name == "v" else (bad, one)), ints([41]))
        for t in q:
            out = bt.cache.attend(q[t], bt.length, row_start=bt.row_start)
            assert torch.equal(out[:40], clean[t][:40]) and torch.equal(out[64:], clean[t][64:])
            assert out[40:64].isnan().all()
    # NaN and infinite queries stay in their own rows and heads
    bt2 = Batch(ops, [70], [10], n_kv=1, hd=64, page=16, seed=3)
    bt2.fill()
    for t in (BF16, F32):
        q = rnd(bt2.rng, 10, 4, 64, dtype=t)
        want = bt2.cache.attend(q, bt2.length, row_start=bt2.row_start)
        q[3, 1, 5], q[7, 2, 0] = float("nan"), float("inf")
        out = bt2.cache.attend(q, bt2.length, row_start=bt2.row_start)
        assert out[3, 1].isnan().all() and out[7, 2].isnan().all()
        for i, h in ((3, 1), (7, 2)):
            out[i, h] = want[i, h] = 0
        assert torch.equal(out, want)


def test_large_pool_offsets(ops):
    """Pages whose blocks lie past 4 GiB of the pool."""
    n_kv, hd, page = 8, 128, 128
    n_pages = (5 << 30) // (2 * n_kv * page * (hd + 4))
    table = ints([[n_pages - 1, 3, n_pages - 2]])
    cache = ops.KvCache.empty(n_pages, n_kv, hd, table, page=page)
    rng = np.random.default_rng(4)
    k, v = (rnd(rng, 300, n_kv, hd) for _ in "kv")
    cache.append(k, v, ints([300]), row_start=ints([0, 300]))
    rk, rv = cache.read(ints([300]), row_start=ints([0, 300]), n_rows=300, dtype=F32)
    K, V = oracle.kv8_values(f64(k)), oracle.kv8_values(f64(v))
    assert np.array_equal(rk.cpu().numpy(), K.astype(np.float32))
    assert np.array_equal(rv.cpu().numpy(), V.astype(np.float32))
    q = rnd(rng, 1, 8, hd)
    bt = Batch.__new__(Batch)
    bt.lens, bt.rows, bt.start = [300], [1], np.array([0])
    check_attend(bt, q, cache.attend(q, ints([300])), [K], [V], hd ** -0.5)


# ------------------------------------------------------------------ together, as they are used
def test_decoding_in_a_graph_on_another_stream(ops):
    """Rotation + append + attention of single tokens captured once and replayed as the
    sequences grow (lengths and page tables change in place), against eager calls; two graphs
    share nothing but the cache."""
    rng = np.random.default_rng(8)
    B, H, G, hd, page = 5, 2, 4, 128, 16
    table = ints([[7 * b + i for i in range(7)] for b in range(B)])
    t = ops.rope_table(200, hd)
    caches = [ops.KvCache.empty(7 * B, H, hd, table, page=page) for _ in "ab"]
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
        for c in caches:                            # warm up on the stream (both: it appends)
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
    # the same on a stream of its own, named in the call
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    qq = caches[0].append(k, v, length, rope=t, q=q, stream=side)
    out = caches[0].attend(qq, length, stream=side)
    side.synchronize()
    assert torch.equal(out, eager)


def test_prompt_then_tokens_is_one_long_prompt(ops):
    """A prompt in chunks and then token by token leaves the cache, and gives the rows, that
    one call does."""
    rng = np.random.default_rng(9)
    n, H, G, hd, page = 150, 2, 4, 64, 32
    table = ints([[4, 0, 3, 1, 2]])
    a, b = (ops.KvCache.empty(5, H, hd, table, page=page) for _ in "ab")
    t = ops.rope_table(n, hd, layout="pairs")
    q, k, v = (rnd(rng, n, x, hd, dtype=F32) for x in (H * G, H, H))
    full = a.attend(a.append(k, v, ints([n]), row_start=ints([0, n]), rope=t, q=q), ints([n]),
                    row_start=ints([0, n]))
    parts = []
    for lo, hi in [(0, 70), (70, 71), (71, 143)] + [(i, i + 1) for i in range(143, n)]:
        at = dict(row_start=ints([0, hi - lo]))
        qq = b.append(k[lo:hi], v[lo:hi], ints([hi]), rope=t, q=q[lo:hi], **at)
        parts.append(b.attend(qq, ints([hi]), **at))
    for x, y in zip(a.read(ints([n]), row_start=ints([0, n]), n_rows=n, dtype=F32),
                    b.read(ints([n]), row_start=ints([0, n]), n_rows=n, dtype=F32)):
        assert torch.equal(x, y)
    # both within the bound of check_attend; rows of unit scale: 2^-17 covers twice that
    assert (torch.cat(parts) - full).abs().max() <= 2.0 ** -17 * 4


def test_prompts_in_a_graph(ops):
    """A packed batch of prompts (its rows padded) captured once for each way of launching it, and
    replayed as rows, lengths and pages change in place, against eager calls."""
    rng = np.random.default_rng(12)
    H, G, hd, page = 4, 8, 128, 16
    for hints in (dict(max_rows=400, max_length=500), dict(max_rows=4, max_length=500),
                  dict(max_rows=400, max_length=30000)):
        table = ints(rng.permutation(96).reshape(2, 48).tolist())
        cache = ops.KvCache.empty(96, H, hd, table, page=page)
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


def test_shared_pages_and_two_streams(ops):
    """Sequences that begin with the same pages (and one page twice in a sequence) attend over
    them at once on two streams, each call with a workspace of its own."""
    bt = Batch(ops, [640], [640], n_kv=2, hd=128, page=16)
    K, V = bt.fill()
    own = bt.table[0, :40]
    shared = torch.stack([own, own.flip(0), own[:1].expand(40)]).contiguous()
    cache = ops.KvCache(bt.cache.pool, shared, page=16, head_dim=128)
    lens = [640, 631, 100]
    where = [np.arange(640), (39 - np.arange(640) // 16) * 16 + np.arange(640) % 16, np.arange(640) % 16]
    sub = Batch.__new__(Batch)
    sub.lens, sub.rows, sub.start = lens, [1, 1, 1], np.arange(4)
    KK, VV = ([x[0][w[:n]] for w, n in zip(where, lens)] for x in (K, V))
    q = [rnd(bt.rng, 3, 8, 128, dtype=F32) for _ in "ab"]
    length = ints(lens)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in "ab"]
    outs = [[cache.attend(x, length, stream=s) for s, x in zip(streams, q)] for _ in range(20)]
    torch.cuda.synchronize()
    for got in outs:
        for x, first, out in zip(q, outs[0], got):
            assert torch.equal(out, first)
            check_attend(sub, x, out, KK, VV, 128 ** -0.5)
    for x, first in zip(q, outs[0]):
        y = x.clone()
        assert cache.attend(y, length, out=y) is y and torch.equal(y, first)   # out may be q


def test_memory_in_use_on_another_stream_is_not_handed_out(ops):
    """A cache or a table dropped while a call on another stream still waits stays allocated
    until that call is done."""
    side = torch.cuda.Stream()
    x = torch.zeros(1, 2, 64, device="cuda")
    one = ints([1])

    def calls():
        cache = ops.KvCache.empty(64, 2, 64, ints([[0]]), page=64)
        table = ops.rope_table(50000, 64)
        kept = [t.data_ptr() for t in (cache.pool, table.cos, table.sin)]
        yield lambda: cache.append(x, x, one, rope=table, stream=side), kept
        cache = ops.KvCache.empty(64, 2, 64, ints([[0]]), page=64)
        yield lambda: cache.read(one, stream=side), [cache.pool.data_ptr()]
        cache = ops.KvCache.empty(64, 2, 64, ints([[0]]), page=64)
        yield lambda: cache.attend(x, one, stream=side), [cache.pool.data_ptr()]
        table = ops.rope_table(50000, 64)
        yield lambda: ops.rope(x, one, table, stream=side), [table.cos.data_ptr(), table.sin.data_ptr()]

    for i in range(4):
        it = calls()
        for _ in range(i + 1):
            call, kept = next(it)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(200_000_000)
        call()
        it.close()
        del it, call
        new = [torch.empty(n, dtype=torch.uint8, device="cuda")
               for n in (64 * 2 * 2 * 64 * 68, 50000 * 32 * 4, 50000 * 32 * 4)]
        busy = not side.query()
        assert busy and not set(kept) & {t.data_ptr() for t in new}, i
        torch.cuda.synchronize()


def test_many_sequences_in_a_part_of_a_wider_table(ops):
    """3000 sequences of none to three new rows each: every row finds its own, in a table whose
    rows are longer than the cache's part of them."""
    rng = np.random.default_rng(31)
    n, H, G, hd, page = 3000, 1, 4, 64, 16
    new = rng.integers(0, 4, n)
    new[:5], new[-3:] = 0, 0
    lens = new + rng.integers(0, 20, n)
    wide = ints(rng.integers(-9, 0, (n, 9)).tolist())
    wide[:, 4:6] = ints(rng.permutation(2 * n).reshape(n, 2).tolist())
    cache = ops.KvCache.empty(2 * n, H, hd, wide[:, 4:6], page=page)
    length = ints(lens.tolist())
    whole = np.concatenate([[0], np.cumsum(lens)])
    k, v = (rnd(rng, int(whole[-1]), H, hd) for _ in "kv")
    cache.append(k, v, length, row_start=ints(whole.tolist()))
    K, V = oracle.kv8_values(f64(k)), oracle.kv8_values(f64(v))
    rk, rv = cache.read(length, row_start=ints(whole.tolist()), n_rows=int(whole[-1]), dtype=F32)
    assert np.array_equal(f64(rk), K.astype(np.float32)) and np.array_equal(f64(rv), V.astype(np.float32))
    bt = Batch.__new__(Batch)
    bt.lens, bt.rows, bt.start = lens.tolist(), new.tolist(), np.concatenate([[0], np.cumsum(new)])
    for dtype in (BF16, F32):
        q = rnd(rng, int(bt.start[-1]), H * G, hd, dtype=dtype)
        out = cache.attend(q, length, row_start=ints(bt.start.tolist()))
        check_attend(bt, q, out, [K[a:b] for a, b in zip(whole, whole[1:])],
                     [V[a:b] for a, b in zip(whole, whole[1:])], 0.125)


def test_keys_past_the_rotary_tables_are_kept_as_nan(ops):
    bt = Batch(ops, [30], [30], n_kv=1, hd=64, page=16)
    t = ops.rope_table(20, 32, layout="pairs")
    k, v = (rnd(bt.rng, 30, 1, 64) for _ in "kv")
    q = bt.cache.append(k, v, bt.length, row_start=bt.row_start, rope=t, q=k.repeat(1, 2, 1))
    rk, rv = bt.cache.read(bt.length, row_start=bt.row_start, n_rows=30, dtype=F32)
    assert not rk[:20].isnan().any() and rk[20:].isnan().all() and not rv.isnan().any()
    assert not q[:20].isnan().any() and q[20:, :, :32].isnan().all() and not q[20:, :, 32:].isnan().any()
    out = bt.cache.attend(k.repeat(1, 2, 1), bt.length, row_start=bt.row_start)
    assert not out[:20].isnan().any() and out[20:].isnan().all()


def test_calls_that_name_the_captured_stream(ops):
    """Capture of calls that name their stream, on the stream that is captured."""
    bt = Batch(ops, [300, 40], n_kv=2, hd=64, page=16)
    bt.fill()
    q, k, v = (rnd(bt.rng, 2, h, 64) for h in (8, 2, 2))
    t = ops.rope_table(400, 64)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def step():
        qq = bt.cache.append(k, v, bt.length, rope=t, q=q, stream=s)
        return bt.cache.attend(qq, bt.length, stream=s)

    with torch.cuda.stream(s):
        want = step().clone()
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out = step()
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_no_sequences(ops):
    """A cache whose table has no sequence takes calls that have no rows."""
    cache = ops.KvCache.empty(2, 2, 64, torch.zeros(0, 3, dtype=torch.int32, device="cuda"), page=16)
    none, x = ints([]).view(0), torch.zeros(0, 2, 64, device="cuda")
    assert cache.append(x, x, none) is None
    assert cache.attend(x, none).shape == (0, 2, 64) and cache.read(none)[0].shape == (0, 2, 64)


def test_workspace_given_and_refused(ops):
    bt = Batch(ops, [3000] * 2, n_kv=1, hd=64, page=64)
    bt.fill()
    q = rnd(bt.rng, 2, 4, 64)
    need = bt.cache.attend_workspace(2, 4, 2)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    assert torch.equal(bt.cache.attend(q, bt.length, workspace=ws), bt.cache.attend(q, bt.length))
    with pytest.raises(Exception, match="WICI_E_ARG"):
        bt.cache.attend(q, bt.length, workspace=ws[:-1])


def test_python_refusals(ops):
    bt = Batch(ops, [5, 6], n_kv=2, hd=64, page=16)
    k = torch.zeros(2, 2, 64, device="cuda")
    q = torch.zeros(2, 4, 64, device="cuda")
    bad = ValueError, TypeError, RuntimeError
    t = ops.rope_table(8, 64)
    for call in (lambda: bt.cache.append(k.half(), k, bt.length),
                 lambda: bt.cache.append(k[:1], k, bt.length),
                 lambda: bt.cache.append(k, k, bt.length.long()),
                 lambda: bt.cache.append(k, k, bt.length[:1]),
                 lambda: bt.cache.append(k, k, bt.length, q=q),
                 lambda: bt.cache.append(k.cpu(), k, bt.length),
                 lambda: bt.cache.append(k.transpose(1, 2), k, bt.length),
                 lambda: bt.cache.append(k, k, bt.length, rope=ops.rope_table(8, 128)),
                 lambda: bt.cache.attend(q[:, :3], bt.length),
                 lambda: bt.cache.attend(q, ints([1, 2, 3])),
                 lambda: bt.cache.attend(q[..., :32], bt.length),
                 lambda: bt.cache.attend(q, bt.length, out=q[:1]),
                 lambda: bt.cache.attend(q, bt.length, row_start=ints([0, 2])),
                 lambda: bt.cache.read(bt.length, n_rows=3),
                 lambda: ops.rope(q, ints([0]), t),
                 lambda: ops.rope(q.cpu(), ints([0, 1]), t),
                 lambda: ops.rope_table(8, 60),
                 lambda: ops.rope_table(8, 64, scaling="none"),
                 lambda: ops.RopeTable(t.cos, t.sin.double()),
                 lambda: ops.KvCache(bt.cache.pool, bt.table, page=32, head_dim=64),
                 lambda: ops.KvCache(bt.cache.pool, bt.table.long(), page=16, head_dim=64)):
        with pytest.raises(bad):
            call()
    assert bt.cache.attend(q[:0], ints([]).view(0)).shape == (0, 4, 64)
