"""The attention over the 8-bit key-value cache at the ends of its range, without a GPU: the
arithmetic of csrc/kv8_layout.h and csrc/kv8_plan.h on the CPU under the address and
undefined-behaviour sanitizers."""

from __future__ import annotations

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GXX = shutil.which("g++")
BIG = 2 ** 31 - 1


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if GXX is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("kv8_range") / "kv8_range")
    subprocess.run([GXX, "-O1", "-g", "-std=c++17", "-Wall", "-Werror",
                    "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I",
                    os.path.join(ROOT, "paper_2608_24204_amd", "csrc"),
                    os.path.join(ROOT, "tests", "native", "kv8_range_harness.cpp"), "-o", exe], check=True)

    def run(questions):
        text = "".join(" ".join(map(str, (list(q) + [0] * 3)[:4])) + "\n" for q in questions)
        r = subprocess.run([exe], input=text, capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stderr[-2000:]
        out = [tuple(map(int, l.split())) for l in r.stdout.splitlines()]
        assert len(out) == len(questions)
        return out

    return run


@pytest.mark.parametrize("hd", [64, 128])
def test_partial_results_are_aligned_and_apart(ask, hd):
    """Outputs are stored 16 bytes at a time and states 8, in a workspace aligned to 16, for odd
    numbers of parts too (one query head, nine splits)."""
    for parts in (1, 2, 5, 9, 27, 128, 2 ** 24 * 128):
        of = sorted({0, min(1, parts - 1), parts // 2, parts - 1})
        got = ask([("part", p, parts, hd) for p in of])
        for p, (out, state, floats) in zip(of, got):
            assert out % 4 == 0 and state % 2 == 0
            assert out == p * hd and out + hd <= got[0][1] <= state
            assert state + 2 <= floats
        states = [g[1] for g in got]
        assert all(b - a >= 2 for a, b in zip(states, states[1:]))


def test_steps_of_the_longest_contexts(ask):
    q = [(n, step) for step in (32, 64) for n in (0, 1, 31, 32, 33, 64, 65, 2 ** 30, BIG - 64, BIG - 63,
                                                  BIG - 32, BIG - 1, BIG)]
    assert [g[0] for g in ask([("steps", *x) for x in q])] == [-(-n // step) for n, step in q]


def test_the_merge_of_as_many_rows_as_a_call_takes(ask):
    """2^24 rows x heads, the most of a call, and any fewer: a grid that covers them, of fewer than
    2^32 work-items (256 a workgroup) along each dimension."""
    n = [1, 2, 40, 2 ** 20 - 1, 2 ** 20, 2 ** 20 + 1, 5 * 10 ** 6, 2 ** 24 - 1, 2 ** 24]
    for rows, (x, y) in zip(n, ask([("merge", r) for r in n])):
        assert 256 * x < 2 ** 32 and 1 <= y <= 65535
        assert x * y >= rows > x * (y - 1)
        assert y == 1 or rows > 2 ** 20
