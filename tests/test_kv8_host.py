"""The 8-bit key-value cache without a GPU: its layout, the bounds its kernels put on page
tables, lengths and row ranges (csrc/kv8_layout.h evaluated on the CPU under the address
and undefined-behaviour sanitizers), and what its entry points refuse before any GPU call."""

from __future__ import annotations

import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

import oracle
from paper_2608_24204_amd import binding
from tests.helpers import small_cfg
from tests.test_gpu_kv8 import PLAN_CASES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GXX = shutil.which("g++")
BIG = 2 ** 31 - 1


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if GXX is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("kv8") / "kv8")
    subprocess.run([GXX, "-O1", "-g", "-std=c++17", "-Wall", "-Werror",
                    "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I",
                    os.path.join(ROOT, "paper_2608_24204_amd", "csrc"),
                    os.path.join(ROOT, "tests", "native", "kv8_harness.cpp"), "-o", exe], check=True)

    def run(questions):
        text = "".join(" ".join(map(str, (list(q) + [0] * 8)[:8])) + "\n" for q in questions)
        r = subprocess.run([exe], input=text, capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stderr[-2000:]
        out = [tuple(map(int, l.split())) for l in r.stdout.splitlines()]
        assert len(out) == len(questions)
        return out

    return run


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_a_block_holds_every_code_once_where_the_definition_says(ask, page, hd):
    size, *at = ask([("block", page, hd)])[0]
    n = page * hd
    keys, values, scales = at[:n], at[n:2 * n], at[2 * n:]
    assert size == n + 4 * page and size % 16 == 0
    rows = np.random.default_rng(page + hd).standard_normal((page, hd)).astype(np.float32)
    kb, vb = oracle.kv8_block(rows)
    codes, steps = oracle.kv8_quantise(rows)
    assert len(kb) == len(vb) == size
    assert np.array_equal(kb[keys], (codes + 128).reshape(-1))
    assert np.array_equal(vb[values], (codes + 128).reshape(-1))
    for want, b in ((steps, kb), (steps, vb)):
        assert np.array_equal(np.stack([b[s:s + 4] for s in scales]).view("<f4")[:, 0], want)
    assert sorted(keys) == sorted(values) == list(range(n))


def test_blocks_follow_each_other_past_32_bits(ask):
    for page, hd, n_kv in ((16, 64, 1), (64, 128, 8), (128, 128, 1024)):
        size = page * (hd + 4)
        q = [(p, w, h) for p in (0, 1, 70000, BIG - 1) for w in (0, 1) for h in (0, n_kv - 1)]
        got = ask([("at", p, w, h, n_kv, page, hd) for p, w, h in q])
        assert [g[0] for g in got] == [((p * 2 + w) * n_kv + h) * size for p, w, h in q]


def test_a_page_is_taken_only_from_inside_the_table_and_the_pool(ask):
    q, want = [], []
    for p in (-1, 0, 3, 4, BIG, -BIG):
        for entry in (-1, 0, 6, 7, BIG, -BIG):
            q.append(("page", p, 4, 7, entry))
            want.append(entry if 0 <= p < 4 and 0 <= entry < 7 else -1)
    assert [a[0] for a in ask(q)] == want


def test_row_ranges_stay_inside_the_rows(ask):
    vals = (-BIG - 1, -3, 0, 1, 5, 9, 10, 11, BIG)
    q = [(f, t, 10) for f in vals for t in vals]
    for (f, t, n), (row0, rows) in zip(q, ask([("range", *x) for x in q])):
        assert 0 <= row0 <= n and rows >= 0 and row0 + rows <= n
        if 0 <= f <= t <= n:
            assert (row0, rows) == (f, t - f)


def test_rows_see_positions_up_to_their_own(ask):
    q = [(length, rows, i, cap) for length in (0, 1, 5, 64, BIG) for rows in (1, 3, 9)
         for i in range(rows) for cap in (16, 64, 2 ** 31)]
    got = ask([("seen", *x) for x in q])
    assert [g[0] for g in got] == [min(max(n - r + i + 1, 0), min(cap, BIG + 1)) for n, r, i, cap in q]


def test_the_oracle_rounds_codes_exactly():
    # 127 x / a = k + 1/2 exactly for a = 254: ties to even
    x = np.array([[254.0, 1.0, 3.0, -1.0, -3.0, 5.0, 0.0, 2.0]], np.float32)
    assert oracle.kv8_quantise(x)[0].tolist() == [[127, 0, 2, 0, -2, 2, 0, 1]]
    n, step = oracle.kv8_quantise(np.zeros((1, 8), np.float32))
    assert not n.any() and step[0] == np.float32(2.0 ** -60 / 127)
    assert np.isnan(oracle.kv8_values(np.array([[1.0, np.inf] * 4]))).all()
    assert np.isnan(oracle.kv8_values(np.array([[1.0, np.nan] * 4]))).all()


def test_the_gpu_tests_meet_every_kernel(ask):
    """The attention's kernels (a split of few rows, tiles of 64 and of 128 rows), with and
    without partial results to merge, for both head sizes and one and two terms."""
    seen = set()
    for n_seqs, rows, length, n_kv, G, hd, entries, page in PLAN_CASES:
        for terms in (1, 2):
            (kind, _, nsplit), = ask([("plan", hd, terms, n_kv * G, n_kv, n_seqs, rows,
                                       entries * page)])
            seen.add((hd, terms, kind, nsplit > 1))
    # (one term: tiles of 64 rows are taken where the chip is half full: nothing is left to
    # split; two terms: never tiles of 128)
    assert seen == {(hd, t, k, s) for hd in (64, 128) for t, k, s in (
        (1, 0, False), (1, 0, True), (1, 1, False), (1, 2, False), (1, 2, True),
        (2, 0, False), (2, 0, True), (2, 1, False), (2, 1, True))}


def test_launch_sizes(ask):
    """Grids within their limits, splits and row tiles that cover the rows, over the range of
    the operator."""
    rng = np.random.default_rng(0)
    q = []
    for _ in range(2000):
        n_kv = int(rng.choice([1, 2, 8, 64]))
        q.append(("plan", int(rng.choice([64, 128])), int(rng.choice([1, 2])),
                  n_kv * int(rng.integers(1, 17)), n_kv, int(2 ** rng.uniform(0, 12)),
                  int(2 ** rng.uniform(0, 16)), int(2 ** rng.uniform(0, 24))))
    q += [("plan", hd, 1, 8, 8, n, 2 ** 24, 2 ** 31 - 1) for hd in (64, 128) for n in (1, 65535)]
    for (_, hd, terms, hq, n_kv, n_seqs, rows, length), (kind, ntile, nsplit) in zip(q, ask(q)):
        per = 64 * kind if kind else 16
        assert kind in (0, 1, 2) and ntile * per >= rows * (hq // n_kv) > (ntile - 1) * per
        assert 1 <= nsplit <= 128
        most = 2 * 256 if kind else 256 * (4 if hd == 64 else 3 if terms == 1 else 2)
        assert nsplit == 1 or nsplit * ntile * n_kv * n_seqs <= most
        assert kind < 2 or terms == 1
    # workspaces are sized for one term's plan: two terms never split further
    for (one,), (two,) in zip(*[[ask([("plan", hd, t, 32, 8, n, r, m)]) for hd in (64, 128)
                                 for n in (1, 3, 20) for r in (1, 40, 333, 2048)
                                 for m in (100, 513, 700, 2000, 9000, 2 ** 31 - 1)] for t in (1, 2)]):
        assert two[2] <= one[2]


# ------------------------------------------------------------------ refusals
FAKE = 1 << 20   # an aligned address that no refused call may touch


def _cache(**kw):
    c = binding.WiciKv8(FAKE, 10, 64, 2, 128, FAKE, 5, 5)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _batch(**kw):
    b = binding.WiciKv8Batch(3, 3, None, FAKE, 0, 0)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def _rows(heads=2, d=128, **kw):
    r = binding.WiciHeadRows(FAKE, binding.WICI_BF16, heads * d, d)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def _tab(**kw):
    t = binding.WiciRopeTab(FAKE, FAKE, 100, 128, 0)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


lib_built = pytest.mark.skipif(not os.path.exists(binding.LIB_PATH), reason="libwici.so not built")
BAD_CACHE = [dict(pool=None), dict(pool=FAKE + 8), dict(n_pages=0), dict(page=48), dict(page=8),
             dict(n_kv_heads=0), dict(head_dim=96), dict(table=None), dict(table_stride=4),
             dict(table_stride=-5), dict(max_pages=0)]
BAD_BATCH = [dict(n_seqs=-1), dict(n_rows=-1), dict(n_rows=4), dict(length=None),
             dict(n_seqs=65536, n_rows=65536), dict(max_rows=-1), dict(max_length=-1)]
BAD_ROWS = [dict(data=None), dict(data=FAKE + 8), dict(dtype=2), dict(dtype=3), dict(row_stride=0),
            dict(row_stride=-256), dict(head_stride=0), dict(head_stride=132), dict(row_stride=260),
            dict(head_stride=64), dict(row_stride=64)]


@lib_built
@pytest.mark.parametrize("cache,batch,rows", [(c, {}, {}) for c in BAD_CACHE] +
                         [({}, b, {}) for b in BAD_BATCH] + [({}, {}, r) for r in BAD_ROWS])
def test_bad_arguments_are_refused(cache, batch, rows):
    lib = binding.load_library()
    c, b = _cache(**cache), _batch(**batch)
    no = binding.WiciHeadRows()
    good, bad = _rows(), _rows(**rows)
    E = binding.WICI_E_ARG
    for k, v in ((bad, good), (good, bad)):
        if bad.data is not None or not rows:
            assert lib.wici_kv8_read(c, b, k, v, None) == E
        assert lib.wici_kv8_append(c, b, None, 0, no, no, k, v, None) == E
        assert lib.wici_kv8_attend(c, b, 2, 0.1, k, v, FAKE, 1 << 40, None) == E


@lib_built
def test_refusals_of_single_calls():
    lib = binding.load_library()
    c, b, no, E = _cache(), _batch(), binding.WiciHeadRows(), binding.WICI_E_ARG
    size = ctypes.c_size_t(7)
    assert lib.wici_kv8_read(c, b, no, no, None) == E
    assert lib.wici_kv8_bytes(None, size) == E and lib.wici_kv8_bytes(c, None) == E
    # queries: need rope, rows and a place to go; rope no wider than the heads
    for args in ((None, 4, _rows(4), _rows(4)), (_tab(), 0, _rows(4), _rows(4)),
                 (_tab(), 4, _rows(4), no), (_tab(dim=136), 4, _rows(4), _rows(4)),
                 (_tab(dim=12), 0, no, no), (_tab(cos_t=None), 0, no, no),
                 (_tab(sin_t=FAKE + 4), 0, no, no), (_tab(n_pos=0), 0, no, no),
                 (_tab(layout=2), 0, no, no)):
        assert lib.wici_kv8_append(c, b, *args, _rows(), _rows(), None) == E
    for heads in (0, -2, 3, 1026):
        assert lib.wici_kv8_attend_workspace(c, b, heads, size) == E
        assert lib.wici_kv8_attend(c, b, heads, 0.1, _rows(4), _rows(4), FAKE, 1 << 40, None) == E
    for scale in (float("nan"), float("inf")):
        assert lib.wici_kv8_attend(c, b, 4, scale, _rows(4), _rows(4), FAKE, 1 << 40, None) == E
    # a workspace that is too small, missing or misaligned
    assert lib.wici_kv8_attend_workspace(c, b, 4, size) == 0 and size.value == 0   # short: no split
    long = _cache(max_pages=50, table_stride=50)
    assert lib.wici_kv8_attend_workspace(long, b, 4, size) == 0 and size.value > 0
    for ws, n in ((FAKE, size.value - 1), (None, size.value), (FAKE + 4, size.value)):
        assert lib.wici_kv8_attend(long, b, 4, 0.1, _rows(4), _rows(4), ws, n, None) == E
    for kw in (dict(head_dim=96), dict(n_rows=-1), dict(n_heads=0), dict(positions=None)):
        a = dict(head_dim=128, n_rows=3, n_heads=2, positions=FAKE) | kw
        assert lib.wici_rope_rows(_tab(), a["head_dim"], a["n_rows"], a["n_heads"], a["positions"],
                                  _rows(), _rows(), None) == E
    # more rows than a call takes
    big = _batch(n_seqs=1, n_rows=1 << 24, row_start=FAKE)
    for heads in (2, 4):
        assert lib.wici_kv8_attend_workspace(c, big, heads, size) == E
        assert lib.wici_kv8_attend(c, big, heads, 0.1, _rows(heads), _rows(heads), FAKE, 1 << 60, None) == E
    wide = _cache(n_kv_heads=8)
    assert lib.wici_kv8_append(wide, big, None, 0, no, no, _rows(8), _rows(8), None) == E
    assert lib.wici_kv8_append(c, big, _tab(), 12, _rows(12), _rows(12), _rows(), _rows(), None) == E
    assert lib.wici_kv8_read(wide, big, _rows(8), no, None) == E
    assert lib.wici_rope_rows(_tab(), 128, 1 << 24, 16, FAKE, _rows(16), _rows(16), None) == E
    for bad in BAD_ROWS:
        assert lib.wici_rope_rows(_tab(), 128, 3, 2, FAKE, _rows(**bad), _rows(), None) == E
        assert lib.wici_rope_rows(_tab(), 128, 3, 2, FAKE, _rows(), _rows(**bad), None) == E
    assert lib.wici_rope_rows(_tab(), 64, 3, 2, FAKE, _rows(d=64), _rows(d=64), None) == E
    assert lib.wici_rope_rows(None, 128, 3, 2, FAKE, _rows(), _rows(), None) == E


@lib_built
@pytest.mark.parametrize("kw", [dict(dim=4), dict(dim=12), dict(dim=136), dict(layout=2),
                                dict(scaling=5), dict(scaling=-1), dict(base=1.0),
                                dict(base=float("inf")), dict(base=float("nan")),
                                dict(scaling=1, factor=0.5), dict(scaling=2, factor=float("nan")),
                                dict(scaling=3, original=0.0), dict(scaling=4, low=2.0, high=1.0),
                                dict(scaling=4, low=0.0, high=8.0)])
def test_bad_rope_specifications_are_refused(kw):
    r = binding.WiciRope(64, 0, 0, 10000.0, 2.0, 2048.0, 0.0, 0.0)
    for k, v in kw.items():
        setattr(r, k, v)
    lib = binding.load_library()
    assert lib.wici_rope_table(ctypes.byref(r), 16, FAKE, FAKE, None) == binding.WICI_E_ARG


@lib_built
def test_nothing_to_do_is_no_error_and_no_gpu_call():
    lib = binding.load_library()
    no, size = binding.WiciHeadRows(), ctypes.c_size_t(7)
    for b in (_batch(n_seqs=0, n_rows=0), _batch(n_rows=0, row_start=FAKE)):
        assert lib.wici_kv8_append(_cache(), b, None, 0, no, no, no, no, None) == 0
        assert lib.wici_kv8_read(_cache(), b, _rows(), no, None) == 0
        assert lib.wici_kv8_attend_workspace(_cache(), b, 4, size) == 0 and size.value == 0
        assert lib.wici_kv8_attend(_cache(), b, 4, 0.1, no, no, None, 0, None) == 0
    b = _batch(n_seqs=0, n_rows=0, length=None)          # a table of no sequences has no address
    assert lib.wici_kv8_append(_cache(table=None), b, None, 0, no, no, no, no, None) == 0
    assert lib.wici_kv8_read(_cache(table=None), b, _rows(), no, None) == 0
    assert lib.wici_kv8_attend(_cache(table=None), b, 4, 0.1, no, no, None, 0, None) == 0
    assert lib.wici_rope_rows(_tab(), 128, 0, 2, None, no, no, None) == 0
    r = binding.WiciRope(64, 0, 0, 10000.0, 0.0, 0.0, 0.0, 0.0)
    assert lib.wici_rope_table(ctypes.byref(r), 0, None, None, None) == 0


@lib_built
def test_pool_size():
    lib, size = binding.load_library(), ctypes.c_size_t()
    assert lib.wici_kv8_bytes(_cache(n_pages=100000, n_kv_heads=8), size) == 0
    assert size.value == 100000 * 2 * 8 * 64 * 132


# ------------------------------------------------------------------ the model's side of it
def _model_cfg(**kw):
    return binding.make_config(small_cfg(**(dict(n_layers=2, d_model=512, n_heads=4, n_kv_heads=2,
                                                 head_dim=128, ffn_dim=512, vocab=1000,
                                                 kv_dtype="kv8") | kw)), max_seq=1000)


@lib_built
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("page", [16, 64])
def test_a_models_cache_has_the_pools_bytes(hd, page):
    c = _model_cfg(head_dim=hd)
    c.kv_page = page
    pages = -(-1000 // page)
    size = ctypes.c_size_t()
    lib = binding.load_library()
    assert lib.wici_kv8_bytes(_cache(n_pages=pages, page=page, n_kv_heads=2, head_dim=hd), size) == 0
    kv = binding.memory_requirements(c)[1]
    assert 2 * size.value <= kv <= 2 * size.value + 4096
    other = _model_cfg(head_dim=hd, kv_dtype="bf16")
    other.kv_page = page
    assert abs(kv / binding.memory_requirements(other)[1] - (hd + 4) / (2 * hd)) < 0.01


@lib_built
def test_set_rope_before_memory_is_bound():
    lib, h = binding.load_library(), ctypes.c_void_p()
    spec = lambda **kw: binding.WiciRope(*(dict(dim=64, layout=1, scaling=3, base=10000.0, factor=2.0,
                                                original=2048.0, low=0.0, high=0.0) | kw).values())
    for kv in ("kv8", "bf16", "f32"):
        c = _model_cfg(head_dim=64, kv_dtype=kv)
        assert lib.wici_create(ctypes.byref(c), None, ctypes.byref(h)) == binding.WICI_OK
        try:
            sizes = binding.memory_requirements(c)
            for bad in (dict(dim=72), dict(dim=128), dict(dim=0), dict(layout=2), dict(scaling=9),
                        dict(base=1.0), dict(factor=0.5), dict(original=-1.0)):
                assert lib.wici_set_rope(h, ctypes.byref(spec(**bad))) == binding.WICI_E_ARG, bad
            assert lib.wici_set_rope(h, None) == binding.WICI_E_ARG
            assert lib.wici_set_rope(None, ctypes.byref(spec())) == binding.WICI_E_ARG
            for good in (dict(), dict(dim=8, layout=0), dict(scaling=0, factor=0.0, original=0.0)):
                assert lib.wici_set_rope(h, ctypes.byref(spec(**good))) == binding.WICI_OK
            assert binding.memory_requirements(c) == sizes
        finally:
            lib.wici_destroy(h)
