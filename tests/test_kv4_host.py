"""The 4-bit key-value cache without a GPU: its layout and scales (csrc/kv4_layout.h evaluated on
the CPU under the address and undefined-behaviour sanitizers), its launch rules, and what its
entry points refuse before any GPU call."""

from __future__ import annotations

import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

import oracle
from paper_2608_24204_amd import binding
from tests.test_gpu_kv8 import PLAN_CASES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GXX = shutil.which("g++")
BIG = 2 ** 31 - 1


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if GXX is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("kv4") / "kv4")
    subprocess.run([GXX, "-O1", "-g", "-std=c++17", "-Wall", "-Werror",
                    "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I",
                    os.path.join(ROOT, "paper_2608_24204_amd", "csrc"),
                    os.path.join(ROOT, "tests", "native", "kv4_harness.cpp"), "-o", exe], check=True)

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
def test_a_block_holds_every_byte_once_where_the_definition_says(ask, page, hd):
    size, *at = ask([("block", page, hd)])[0]
    n, m = page * hd // 2, page * hd // 32
    keys, values, kscale, vscale = at[:n], at[n:2 * n], at[2 * n:2 * n + m], at[2 * n + m:]
    assert size == n + m and size % 16 == 0
    rows = np.random.default_rng(page + hd).standard_normal((page, hd)).astype(np.float32)
    kb, vb = oracle.kv4_block(rows)
    code, byte = oracle.kv4_quantise(rows)
    pairs = (code[:, 0::2] + 16 * code[:, 1::2]).reshape(-1)
    assert len(kb) == len(vb) == size
    assert np.array_equal(kb[keys], pairs) and np.array_equal(vb[values], pairs)
    assert np.array_equal(kb[kscale], byte.reshape(-1)) and np.array_equal(vb[vscale], byte.reshape(-1))
    assert sorted(keys + kscale) == sorted(values + vscale) == list(range(size))


def test_blocks_follow_each_other_past_32_bits(ask):
    for page, hd, n_kv in ((16, 64, 1), (64, 128, 8), (128, 128, 1024)):
        size = page * (hd // 2 + hd // 32)
        q = [(p, w, h) for p in (0, 1, 70000, BIG - 1) for w in (0, 1) for h in (0, n_kv - 1)]
        got = ask([("at", p, w, h, n_kv, page, hd) for p, w, h in q])
        assert [g[0] for g in got] == [((p * 2 + w) * n_kv + h) * size for p, w, h in q]


def test_scales_are_the_least_powers_of_two_that_hold_a_group(ask):
    rng = np.random.default_rng(1)
    x = np.abs(np.concatenate([
        2.0 ** rng.uniform(-149, 128, 3000), *[7 * 2.0 ** rng.integers(-130, 126, 200) * f for f in (1, 1 + 2 ** -23, 1 - 2 ** -23)],
        [0.0, 2.0 ** -149, 3.4028234663852886e38]]).clip(0, 3.4028234663852886e38)).astype(np.float32)
    got = [a[0] for a in ask([("scale", int(b)) for b in x.view(np.uint32)])]
    for v, byte in zip(x.astype(np.float64), got):
        assert 67 <= byte <= 252
        assert byte == 252 or v <= 7.0 * 2.0 ** (byte - 127)
        assert byte == 67 or v > 7.0 * 2.0 ** (byte - 128)
    rows = np.zeros((len(x), 32), np.float32)
    rows[:, 5] = -x
    assert oracle.kv4_quantise(rows)[1][:, 0].tolist() == got


def test_launch_sizes(ask):
    """Grids within their limits, splits and row tiles that cover the rows, over the range of
    the operator; a workspace sized for bf16 rows is enough for the others."""
    rng = np.random.default_rng(0)
    q = []
    for _ in range(2000):
        n_kv = int(rng.choice([1, 2, 8, 64]))
        q.append((int(rng.choice([64, 128])), n_kv * int(rng.integers(1, 17)), n_kv,
                  int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 16)), int(2 ** rng.uniform(0, 24))))
    q += [(hd, 8, 8, n, 2 ** 24, BIG) for hd in (64, 128) for n in (1, 65535)]
    both = [ask([("plan", hd, t, hq, n_kv, n, r, m) for hd, hq, n_kv, n, r, m in q]) for t in (1, 3)]
    for (hd, hq, n_kv, n_seqs, rows, length), one, three in zip(q, *both):
        assert three[2] <= one[2]
        for terms, (kind, ntile, nsplit) in ((1, one), (3, three)):
            per = 64 * kind if kind else 16
            assert kind in (0, 1, 2) and ntile * per >= rows * (hq // n_kv) > (ntile - 1) * per
            assert 1 <= nsplit <= 128 and ntile * nsplit * n_kv <= BIG
            assert kind < 2 or terms == 1


# ------------------------------------------------------------------ refusals
FAKE = 1 << 20   # an aligned address that no refused call may touch


def test_refusals():
    lib = binding.load_library()
    rows = binding.WiciHeadRows(FAKE, binding.WICI_BF16, 256, 128)
    size = ctypes.c_size_t()

    def cache(**kw):
        c = binding.WiciKv8(FAKE, 10, 64, 2, 128, FAKE, 5, 5)
        for k, v in kw.items():
            setattr(c, k, v)
        return c

    def batch(**kw):
        b = binding.WiciKv8Batch(3, 3, None, FAKE, 0, 0)
        for k, v in kw.items():
            setattr(b, k, v)
        return b

    assert lib.wici_kv4_bytes(cache(), ctypes.byref(size)) == 0 and size.value == 10 * 2 * 2 * 64 * 68
    for bad in (dict(head_dim=96), dict(page=48), dict(n_pages=0), dict(n_kv_heads=0)):
        assert lib.wici_kv4_bytes(cache(**bad), ctypes.byref(size)) == binding.WICI_E_ARG
    assert lib.wici_kv4_bytes(None, ctypes.byref(size)) == binding.WICI_E_ARG
    none = binding.WiciHeadRows()
    odd = binding.WiciHeadRows(FAKE + 8, binding.WICI_BF16, 256, 128)
    narrow = binding.WiciHeadRows(FAKE, binding.WICI_BF16, 256, 124)
    other = binding.WiciHeadRows(FAKE, binding.WICI_KV8, 256, 128)
    for c, b, k in ((cache(pool=FAKE + 4), batch(), rows), (cache(max_pages=0), batch(), rows),
                    (cache(), batch(n_rows=4), rows), (cache(), batch(length=None), rows),
                    (cache(), batch(), none), (cache(), batch(), odd), (cache(), batch(), narrow),
                    (cache(), batch(), other), (cache(table_stride=4), batch(), rows),
                    (cache(), batch(n_seqs=65536, n_rows=65536), rows)):
        assert lib.wici_kv4_append(c, b, None, 0, none, none, k, rows, None) == binding.WICI_E_ARG
        assert lib.wici_kv4_read(c, b, k, none, None) == binding.WICI_E_ARG
        assert lib.wici_kv4_attend(c, b, 4, 1.0, k, rows, None, 0, None) == binding.WICI_E_ARG
    assert lib.wici_kv4_append(cache(), batch(), None, 4, rows, rows, rows, rows, None) == binding.WICI_E_ARG
    for heads, scale in ((3, 1.0), (0, 1.0), (1026, 1.0), (4, float("nan")), (4, float("inf"))):
        assert lib.wici_kv4_attend(cache(), batch(), heads, scale, rows, rows, None, 0,
                                   None) == binding.WICI_E_ARG
    # a workspace too small or not there
    assert lib.wici_kv4_attend_workspace(cache(max_pages=300, table_stride=300),
                                         batch(n_seqs=1, n_rows=1), 4, ctypes.byref(size)) == 0
    assert size.value > 0
    assert lib.wici_kv4_attend(cache(max_pages=300, table_stride=300), batch(n_seqs=1, n_rows=1), 4, 1.0,
                               rows, rows, None, size.value, None) == binding.WICI_E_ARG
    assert lib.wici_kv4_attend(cache(max_pages=300, table_stride=300), batch(n_seqs=1, n_rows=1), 4, 1.0,
                               rows, rows, FAKE, size.value - 1, None) == binding.WICI_E_ARG
    # calls without rows do nothing
    for b in (batch(n_seqs=0, n_rows=0), ):
        assert lib.wici_kv4_append(cache(), b, None, 0, none, none, none, none, None) == 0
        assert lib.wici_kv4_attend(cache(), b, 4, 1.0, none, none, None, 0, None) == 0


def test_the_gpu_tests_meet_every_kernel(ask):
    """The attention's kernels (a split of few rows, of one tile of them or more; tiles of 64 and of 128
    rows), with and without partial results to merge, for both head sizes, bf16 and other rows."""
    seen = set()
    for n_seqs, rows, length, n_kv, G, hd, entries, page in PLAN_CASES:
        for terms in (1, 3):
            (kind, ntile, nsplit), = ask([("plan", hd, terms, n_kv * G, n_kv, n_seqs, rows, entries * page)])
            seen.add((hd, terms, kind, nsplit > 1, ntile > 1 if kind == 0 else None))
    # (tiles of 64 rows of bf16 are taken where the chip is half full: nothing is left to split)
    assert seen == {(hd, t, k, s, m) for hd in (64, 128) for t, k, s, m in (
        (1, 0, False, True), (1, 0, True, False), (1, 1, False, None), (1, 2, False, None), (1, 2, True, None),
        (3, 0, False, True), (3, 0, True, False), (3, 1, False, None), (3, 1, True, None))}
