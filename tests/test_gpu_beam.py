"""A beam search's selection and the reordering of paged caches against their definitions
(oracle/beam.py).

Tolerances.  Beams, words, page numbers and copied bytes have one right answer.  A score is formed in
64 bits, with exponentials within 2^-34 of themselves and so a logarithm of their sum within 2^-33, and
rounded to fp32 once: |s| 2^-24 + 2^-33 + |s| 2^-50."""

from __future__ import annotations

import numpy as np
import pytest

import oracle
from tests.test_gpu_kv4 import Batch4, sub_batch, tolerance  # noqa: F401
from tests.test_gpu_kv8 import BF16, F32, f64, ints, ops, rnd  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def check_select(ops, logits, scores, k, **kw):
    got = ops.beam_select(logits, scores, k, **kw)
    n, beams = scores.shape
    assert [tuple(x.shape) for x in got] == [(n, k)] * 3
    assert [x.dtype for x in got] == [F32, torch.int32, torch.int32]
    compare(got, logits, scores, k)
    return got


def compare(got, logits, scores, k):
    n, beams = scores.shape
    z, c = f64(logits).reshape(n, beams, -1), f64(scores)
    s, p, v = (x.cpu().numpy() for x in got)
    for b in range(n):
        ws, wp, wv = oracle.beam_select(z[b], c[b], k)
        assert np.array_equal(p[b], wp) and np.array_equal(v[b], wv), (b, p[b], wp, v[b], wv)
        fine = np.isfinite(ws)
        assert np.array_equal(s[b][~fine], ws[~fine], equal_nan=True)
        err = np.abs(s[b][fine].astype(np.float64) - ws[fine])
        assert (err <= np.abs(ws[fine]) * (2.0 ** -24 + 2.0 ** -50) + 2.0 ** -33).all()


# ------------------------------------------------------------------ selection
@pytest.mark.parametrize("vocab", [1, 2, 7, 63, 64, 65, 255, 1000, 4097, 50257, 152064])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,beams,k", [(1, 1, 1), (3, 4, 8), (2, 7, 7), (1, 16, 64), (1, 64, 33)])
def test_select(ops, vocab, dtype, n, beams, k):
    rng = np.random.default_rng(vocab + beams)
    z = rnd(rng, n * beams, vocab, dtype=dtype, scale=3.0)
    c = rnd(rng, n, beams, dtype=F32, scale=2.0) - 20
    check_select(ops, z, c, k)
    assert ops.beam_select(z, c)[0].shape == (n, beams)      # as many as beams


@pytest.mark.parametrize("vocab,dtype", [(300001, F32), ((1 << 21) + 3, BF16), (1 << 24, BF16), ((1 << 24) - 1, F32)])
def test_select_from_large_vocabularies(ops, vocab, dtype):
    """Groups of several loads, of as many as a unit's and more."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    z = 3 * torch.randn(2, vocab, device="cuda", generator=g)
    check_select(ops, z.to(dtype), torch.tensor([[-3.0, -2.5]], device="cuda"), 20)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [5, 130, 3001])
def test_select_from_rows_of_any_alignment(ops, dtype, vocab):
    rng = np.random.default_rng(vocab)
    for off in range(9):
        wide = rnd(rng, 6, vocab + 11 + off, dtype=dtype, scale=2.0)
        wide[:, :off], wide[:, off + vocab:] = NAN, 1e30     # around the rows
        check_select(ops, wide[:, off:off + vocab], torch.zeros(2, 3, device="cuda"), 5)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_ties_go_to_the_lowest_beam_and_word(ops, dtype):
    for vocab in (64, 3000, 40000):
        flat = torch.zeros(4, vocab, dtype=dtype, device="cuda")
        flat[1, 1::2] = -0.0                                 # equal to zero
        flat[3] = flat[2] + 4                                # the same probabilities
        s, p, v = check_select(ops, flat, torch.tensor([[-1.0] * 4], device="cuda"), 64)
        assert (p == 0).all() and v[0].tolist() == list(range(64))
        s, p, v = check_select(ops, flat, torch.tensor([[-INF, -1, -1, -1]], device="cuda"), 40)
        assert (p == 1).all() and v[0].tolist() == list(range(40))
    rng = np.random.default_rng(2)
    few = torch.from_numpy(rng.integers(0, 4, (6, 5000)).astype(np.float32)).to(dtype).cuda()
    few[3:] = few[:3]                                        # beams that are alike
    check_select(ops, few, torch.tensor([[-1.0, -2, -3, -1, -2, -3]], device="cuda"), 64)
    # the last words alone
    last = torch.full((2, 7001), -3.0, dtype=dtype, device="cuda")
    last[:, -5:] = 1
    s, p, v = check_select(ops, last, torch.tensor([[0.0, 0.0]], device="cuda"), 12)
    assert v[0, :10].tolist() == list(range(6996, 7001)) * 2


def test_words_and_beams_that_are_out(ops):
    rng = np.random.default_rng(3)
    for dtype in (BF16, F32):
        z = rnd(rng, 12, 900, dtype=dtype, scale=2.0)
        z[0, :] = -INF                                       # no word at all
        z[1, 3:] = -INF
        z[2, :899] = -INF
        z[5] = NAN                                           # not alive, below
        z[6], z[7, 5] = INF, NAN
        c = torch.tensor([[-1.0, -2, -3, -9], [-1, -INF, -INF, -INF], [-INF] * 4], device="cuda")
        for k in (1, 4, 30):
            s, p, v = check_select(ops, z, c, k)
            assert not (p[0] == 0).any() and (p[1] == 0).all()
            assert (p[2] == -1).all() and (v[2] == -1).all() and (s[2] == -INF).all()
        z[:4, 4:] = -INF                                     # fewer than k in all
        s, p, v = check_select(ops, z, c, 10)
        assert (p[0, 7:] == -1).all() and (s[0, 7:] == -INF).all() and (p[0, :7] >= 0).all()
        # a NaN or an infinity in what is alive
        for bad in (z.clone(), z.clone(), z.clone()):
            bad[5] = 0
            bad[8:] = 0
            bad[10, 899] = INF if bad is not z else 0
            got = check_select(ops, bad, torch.zeros(3, 4, device="cuda"), 4)
            assert got[0][1].isnan().all() and (got[1][2] == -1).all()
        for c2 in (NAN, INF):
            got = check_select(ops, z[:4], torch.tensor([[-1.0, c2, -2, -3]], device="cuda"), 4)
            assert got[0].isnan().all() and (got[1] == -1).all() and (got[2] == -1).all()


def test_scores_nearer_each_other_than_32_bits_tell(ops):
    """Two beams of the same score but for a word of 2^-33 of the probability: the beam without it
    comes first throughout, wherever it lies."""
    rng = np.random.default_rng(4)
    z = rnd(rng, 1, 20000, dtype=F32).expand(2, 20000).contiguous()
    z[:, 777] = -INF
    for i in (0, 1):
        y = z.clone()
        y[i, 777] = float(torch.logsumexp(z[0].double(), 0)) - 33 * 0.6931
        s, p, v = check_select(ops, y, torch.tensor([[-30.0, -30.0]], device="cuda"), 10)
        assert p[0].tolist() == [1 - i, i] * 5


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_logits_of_any_magnitude(ops, dtype):
    rng = np.random.default_rng(5)
    for size in (0.0, 1e-30, 100.0, 1e4, 1e30):
        z = rnd(rng, 6, 9000, dtype=F32, scale=1.0)
        z = (z * size + (50 if size == 1e-30 else 0)).clamp(-3e38, 3e38).to(dtype)
        check_select(ops, z, rnd(rng, 2, 3, dtype=F32), 17)
    falling = torch.linspace(0, -5000, 30000, device="cuda").expand(2, 30000).to(dtype)
    for z in (falling.contiguous(), falling.flip(1).contiguous()):     # the largest first, and last
        check_select(ops, z, torch.zeros(1, 2, device="cuda"), 64)


def test_select_in_a_graph_and_on_two_streams(ops):
    """Captured and replayed as logits and scores change in place; calls at once with a workspace each,
    whose contents do not matter."""
    rng = np.random.default_rng(6)
    z, c = rnd(rng, 20, 30000, dtype=F32), rnd(rng, 5, 4, dtype=F32)
    need = ops.beam_workspace(5, 4, 30000, F32, 8)
    spaces = [torch.full((need,), 255, dtype=torch.uint8, device="cuda") for _ in "abc"]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ops.beam_select(z, c, 8, workspace=spaces[0])
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out = ops.beam_select(z, c, 8, workspace=spaces[0])
    for i in range(4):
        z.copy_(rnd(rng, 20, 30000, dtype=F32))
        c.copy_(rnd(rng, 5, 4, dtype=F32))
        eager = ops.beam_select(z, c, 8)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager))
    compare(eager, z, c, 8)
    side = [torch.cuda.Stream() for _ in "ab"]
    got = [ops.beam_select(z, c, 8, workspace=w, stream=t) for _ in range(10) for t, w in zip(side, spaces[1:])]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for x in got for a, b in zip(x, eager))


def test_select_refusals(ops):
    z, c = torch.zeros(6, 50, device="cuda"), torch.zeros(2, 3, device="cuda")
    assert ops.beam_select(z[:0], c[:0], 5)[1].shape == (0, 5)
    need = ops.beam_workspace(2, 3, 50, F32, 3)
    for call in (lambda: ops.beam_select(z.half(), c), lambda: ops.beam_select(z.cpu(), c),
                 lambda: ops.beam_select(z, c.cpu()), lambda: ops.beam_select(z, c.double()),
                 lambda: ops.beam_select(z[:5], c), lambda: ops.beam_select(z.t().contiguous().t(), c),
                 lambda: ops.beam_select(z, c, 0), lambda: ops.beam_select(z, c, 65),
                 lambda: ops.beam_select(z[:1].expand(6, 50), c),
                 lambda: ops.beam_select(z, c.t().contiguous().t()),
                 lambda: ops.beam_select(z[:, :0], c),
                 lambda: ops.beam_select(torch.zeros(65, 4, device="cuda"), torch.zeros(1, 65, device="cuda")),
                 lambda: ops.beam_select(z.clone().requires_grad_(), c),
                 lambda: ops.beam_select(z, c, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            call()


# ------------------------------------------------------------------ reordering
def make_caches(ops, rng, n, beams, entries, n_kv, hd, page, bits, layers, wide=0):
    seqs = n * beams
    n_pages = seqs * (entries + 1) + 2
    order = rng.permutation(n_pages)
    table = torch.full((seqs, entries + wide), 7, dtype=torch.int32, device="cuda")
    table = table[:, wide // 2:wide // 2 + entries]
    table.copy_(ints(order[:seqs * entries].reshape(seqs, entries).tolist()))
    spare = ints(order[seqs * entries:seqs * (entries + 1)].tolist())
    caches = [ops.KvCache.empty(n_pages, n_kv, hd, table, page=page, bits=bits) for _ in range(layers)]
    for c in caches:
        c.pool.copy_(torch.from_numpy(rng.integers(0, 256, tuple(c.pool.shape), dtype=np.uint8)))
    return caches, table, spare


def check_reorder(ops, caches, parent, length, spare, page, **kw):
    table = caches[0].table
    pools = [c.pool.cpu().numpy() for c in caches]
    want_t, want_s = table.cpu().numpy(), spare.cpu().numpy()
    oracle.beam_reorder(pools, want_t, parent.cpu().numpy(), length.cpu().numpy(), want_s, page)
    assert ops.beam_reorder(caches, parent, length, spare, **kw) is None
    torch.cuda.synchronize()
    assert np.array_equal(table.cpu().numpy(), want_t) and np.array_equal(spare.cpu().numpy(), want_s)
    for c, p in zip(caches, pools):
        assert np.array_equal(c.pool.cpu().numpy(), p)


@pytest.mark.parametrize("n,beams,entries,n_kv,hd,page,bits,layers,wide", [
    (1, 1, 3, 1, 64, 16, 4, 1, 0), (3, 4, 5, 2, 128, 16, 4, 2, 0), (2, 5, 4, 1, 64, 64, 8, 1, 3),
    (1, 64, 3, 1, 64, 16, 4, 1, 0), (4, 2, 140, 1, 64, 16, 8, 1, 2), (2, 3, 2, 3, 128, 128, 4, 70, 0)])
def test_reorder(ops, n, beams, entries, n_kv, hd, page, bits, layers, wide):
    """Every kind of length, parents in every order (each other's, one for all, none), again and
    again on the same pages."""
    rng = np.random.default_rng(beams + entries)
    caches, table, spare = make_caches(ops, rng, n, beams, entries, n_kv, hd, page, bits, layers, wide)
    cap = entries * page
    for step, at in enumerate([page + 3, page + 4, 0, 1, page, cap - 1, cap, cap + 5, -3]):
        lens = [at] * (n * beams) if step != 1 else [at + b for b in range(n) for _ in range(beams)]
        lens = [x if i % beams == 0 else x + 1 for i, x in enumerate(lens)]   # (the first counts)
        parent = rng.integers(0, beams, (n, beams))
        if step == 3:
            parent[:] = (np.arange(beams) + 1) % beams       # around
        if step == 4:
            parent[0] = rng.choice([-1, beams, 2 ** 31 - 1, -2 ** 31], beams)
        if step == 5:
            parent[:] = beams - 1
        check_reorder(ops, caches, ints(parent.tolist()), ints(lens), spare, page)
        # as long as contexts grow, no page belongs to two beams' partial ends, or to a beam and a
        # spare (later steps go back into pages that were full, and so shared)
        if step < 2:
            ends = table.cpu().numpy()[:, 1]
            assert len(set(ends) | set(spare.tolist())) == 2 * n * beams


def test_reorder_with_pages_that_are_absent(ops):
    rng = np.random.default_rng(9)
    caches, table, spare = make_caches(ops, rng, 2, 3, 4, 1, 64, 16, 4, 1)
    table[0, 1], table[1, 0], table[4, 1], spare[2], spare[3] = -1, 10 ** 6, -2 ** 31, -5, 2 ** 31 - 1
    check_reorder(ops, caches, ints([[2, 0, 1], [1, 2, 1]]), ints([20] * 6), spare, 16)
    check_reorder(ops, caches, ints([[1, 1, 0], [0, 0, 0]]), ints([21] * 6), spare, 16)


def test_reorder_of_pages_past_32_bits_of_bytes(ops):
    n_pages = (5 << 30) // (2 * 8 * 128 * 68)
    table = ints([[n_pages - 1], [n_pages - 2]])
    cache = ops.KvCache.empty(n_pages, 8, 128, table, page=128, bits=4)
    for i in (1, 2, 3, 4):
        cache.pool[n_pages - i] = 10 * i
    spare = ints([n_pages - 3, n_pages - 4])
    ops.beam_reorder(cache, ints([[1, 0]]), ints([5, 5]), spare)
    assert [int(x) for x in table[:, 0]] == [n_pages - 3, n_pages - 4]
    assert spare.tolist() == [n_pages - 1, n_pages - 2]
    for i, v in ((1, 10), (2, 20), (3, 20), (4, 10)):
        assert (cache.pool[n_pages - i] == v).all()
    assert cache.pool[:3].numel() and not (cache.pool[0] == 20).all()


def test_reorder_refusals(ops):
    rng = np.random.default_rng(1)
    caches, table, spare = make_caches(ops, rng, 2, 2, 2, 1, 64, 16, 4, 2)
    other = ops.KvCache.empty(caches[0].pool.shape[0], 1, 64, table.clone(), page=16, bits=4)
    p, n = ints([[0, 1], [1, 0]]), ints([5] * 4)
    before = table.clone()
    for call in (lambda: ops.beam_reorder([], p, n, spare), lambda: ops.beam_reorder([caches[0], other], p, n, spare),
                 lambda: ops.beam_reorder(caches, p.long(), n, spare), lambda: ops.beam_reorder(caches, p.view(-1), n, spare),
                 lambda: ops.beam_reorder(caches, p, n[:3], spare), lambda: ops.beam_reorder(caches, p, n, spare.cpu()),
                 lambda: ops.beam_reorder(caches, ints([[0] * 65]), n, spare),
                 lambda: ops.beam_reorder(caches, ints([[0, 1]] * 3), ints([5] * 6), ints([0] * 6))):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            call()
    assert torch.equal(table, before)
    ops.beam_reorder(caches, p[:0], n[:0], spare[:0])        # no searches: nothing


# ------------------------------------------------------------------ together, as they are used
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("graph", [False, True])
def test_a_beam_search_over_two_layers(ops, bits, graph):
    """Append with rotation, attention, selection and reordering, step after step across page ends,
    eager and as one replayed graph: every beam's cache is that of its own words, and each choice
    the definition's of the logits of that step."""
    rng = np.random.default_rng(11)
    n, beams, H, G, hd, page, vocab, steps = 2, 3, 2, 2, 64, 16, 500, 40
    seqs, entries = n * beams, 4
    values = oracle.kv4_values if bits == 4 else oracle.kv8_values
    embed = [rnd(rng, vocab, (G * H + 2 * H) * hd, dtype=F32) for _ in range(2)]
    head = rnd(rng, G * H * hd, vocab, dtype=F32, scale=0.4)
    rope = ops.rope_table(steps + 1, hd)
    table = torch.full((seqs, entries), -1, dtype=torch.int32, device="cuda")
    # every beam a page for each part of its context, and a spare
    table.copy_(ints(rng.permutation(seqs * entries).reshape(seqs, entries).tolist()))
    own = table.clone()
    spare = ints((seqs * entries + np.arange(seqs)).tolist())
    caches = [ops.KvCache.empty(seqs * (entries + 1), H, hd, table, page=page, bits=bits) for _ in range(2)]
    for c in caches:
        c.pool.zero_()
    length = torch.zeros(seqs, dtype=torch.int32, device="cuda")
    token = ints(rng.integers(0, vocab, n).repeat(beams).tolist())
    scores = torch.tensor([[0.0] + [-INF] * (beams - 1)] * n, device="cuda")
    logits = torch.zeros(seqs, vocab, device="cuda")
    parent = torch.zeros(n, beams, dtype=torch.int32, device="cuda")
    before = torch.zeros_like(scores)
    outs = [torch.zeros(seqs, G * H, hd, device="cuda") for _ in caches]

    def step():
        length.add_(1)
        total = 0
        for layer, c in enumerate(caches):
            x = embed[layer][token.long()].view(seqs, -1, hd)
            q = c.append(x[:, G * H:G * H + H], x[:, G * H + H:], length, rope=rope, q=x[:, :G * H])
            c.attend(q, length, out=outs[layer], max_length=steps)
            total = total + outs[layer].reshape(seqs, -1)
        logits.copy_(total @ head)
        before.copy_(scores)
        s, p, t = ops.beam_select(logits, scores)
        scores.copy_(s), parent.copy_(p), token.copy_(t.view(-1))
        ops.beam_reorder(caches, p, length, spare)

    start = token.clone()
    if graph:
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step()
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            step()
        # as it was
        table.copy_(own), spare.copy_(ints((seqs * entries + np.arange(seqs)).tolist()))
        length.zero_(), token.copy_(start)
        scores.copy_(torch.tensor([[0.0] + [-INF] * (beams - 1)] * n, device="cuda"))
        for c in caches:
            c.pool.zero_()
        torch.cuda.synchronize()
        step_ = g.replay
    else:
        step_ = step
    words = [[int(t)] for t in token.tolist()]
    tables = (rope.cos.cpu().numpy(), rope.sin.cpu().numpy())
    emb = [e.cpu().numpy() for e in embed]
    for i in range(steps):
        step_()
        torch.cuda.synchronize()
        for b in range(n):
            ws, wp, wv = oracle.beam_select(f64(logits[b * beams:(b + 1) * beams]), f64(before[b]), beams)
            assert parent[b].tolist() == wp.tolist() and token.view(n, beams)[b].tolist() == wv.tolist()
        for layer in range(2):
            for sq in range(seqs) if i % 7 == 0 or i > steps - 3 else ():
                x = emb[layer][words[sq]].reshape(i + 1, -1, hd)
                c, sn = (y[:i + 1] for y in tables)
                q, k = (oracle.rope_pairs(y, c, sn, "half") for y in (x[:, :G * H], x[:, G * H:G * H + H]))
                K, V = values(k), values(x[:, G * H + H:])
                want, mag, dots = oracle.attend_rows(q[-1:].astype(np.float64), K, V,
                                                     np.ones((1, i + 1), bool), hd ** -0.5)
                # (fp32 rows over either cache: the wider of the two bounds)
                tol = tolerance(want, mag, dots, i + 1, False, F32) + mag * 2.0 ** -21 * (1 + 2 * dots[..., None])
                assert np.all(np.abs(f64(outs[layer][sq:sq + 1]) - want) <= tol), (i, layer, sq)
        words = [words[b * beams + int(parent[b, j])] + [int(token[b * beams + j])]
                 for b in range(n) for j in range(beams)]
        # what a beam's cache holds is that of its words (the new word is not yet in it)
        if i in (15, 16, 33):
            rs = ints((np.arange(seqs + 1) * (i + 1)).tolist())
            for layer, c in enumerate(caches):
                rk, rv = c.read(length, row_start=rs, n_rows=seqs * (i + 1), dtype=F32)
                for sq in range(seqs):
                    x = emb[layer][words[sq][:-1]].reshape(i + 1, -1, hd)
                    k = oracle.rope_pairs(x[:, G * H:G * H + H], *(y[:i + 1] for y in tables), "half")
                    at = slice(sq * (i + 1), (sq + 1) * (i + 1))
                    assert np.array_equal(f64(rk[at]), values(k).astype(np.float32))
                    assert np.array_equal(f64(rv[at]), values(x[:, G * H + H:]).astype(np.float32))


def test_scores_written_in_place(ops):
    """The C call with its scores as output, as a captured search step may keep them."""
    from paper_2608_24204_amd import binding
    rng = np.random.default_rng(21)
    z, c = rnd(rng, 20, 5000, dtype=BF16), rnd(rng, 5, 4, dtype=F32)
    want = ops.beam_select(z, c)
    p, t = (torch.empty(5, 4, dtype=torch.int32, device="cuda") for _ in "pt")
    ws = torch.empty(ops.beam_workspace(5, 4, 5000, BF16, 4), dtype=torch.uint8, device="cuda")
    s = torch.cuda.current_stream()
    st = binding.load_library().wici_beam_select(
        z.data_ptr(), binding.WICI_BF16, 5000, 5, 4, 5000, c.data_ptr(), 4, c.data_ptr(), p.data_ptr(),
        t.data_ptr(), ws.data_ptr(), ws.numel(), s.cuda_stream)
    assert st == 0
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((c, p, t), want))


def test_reordering_on_a_named_stream_and_in_a_graph(ops):
    """Captured once and replayed as lengths and parents change in place; two layers of 8 bits."""
    rng = np.random.default_rng(22)
    caches, table, spare = make_caches(ops, rng, 3, 4, 4, 2, 64, 16, 8, 2)
    other, table2, spare2 = make_caches(ops, np.random.default_rng(22), 3, 4, 4, 2, 64, 16, 8, 2)
    parent, length = ints([[0] * 4] * 3), ints([5] * 12)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    ops.beam_reorder(caches, parent, length, spare, stream=s)
    ops.beam_reorder(other, parent, length, spare2)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        ops.beam_reorder(caches, parent, length, spare)
    for at in (6, 16, 17, 40, 64):
        parent.copy_(ints(rng.integers(-1, 5, (3, 4)).tolist()))
        length.fill_(at)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        ops.beam_reorder(other, parent, length, spare2)
        torch.cuda.synchronize()
        assert torch.equal(table, table2) and torch.equal(spare, spare2)
        assert all(torch.equal(a.pool, b.pool) for a, b in zip(caches, other))
