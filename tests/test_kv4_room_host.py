"""Sums of weighted values in the attention over the 4-bit cache stay within fp32: the bounds of
csrc/kv4_layout.h in exact arithmetic, for contexts of any length."""

from __future__ import annotations

import os
import shutil
import subprocess
from fractions import Fraction

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GXX = shutil.which("g++")


def test_sums_stay_within_fp32(tmp_path):
    if GXX is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path / "room")
    subprocess.run([GXX, "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "paper_2608_24204_amd", "csrc"),
                    os.path.join(ROOT, "tests", "native", "kv4_room_harness.cpp"), "-o", exe], check=True)
    ns = sorted({max(0, min(2 ** 31 - 1, 2 ** i + d)) for i in range(32) for d in (-2, -1, 0, 1, 33)})
    r = subprocess.run([exe], input="\n".join(map(str, ns)), capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stderr[-2000:]
    # a lane's eight weights of a step of 32 positions sum up to `most` at the most, so the four lanes' of a
    # row to four times that
    limit = Fraction(2) ** 128 - Fraction(2) ** 104
    for n, line in zip(ns, r.stdout.splitlines()):
        for i in range(2):
            most, top, log_most, byte, lift = (float(x) for x in line.split()[5 * i:5 * i + 5])
            assert most == 2.0 ** log_most and top < log_most
            weights = -(-n // 32) * 4 * Fraction(most)
            # the largest value that is not large, and joins by factors of at most 1
            assert weights * 6 * Fraction(2) ** int(byte - 1 - 127) < limit / 2
            # the largest value, lifted, and two joins by less than 2 each
            assert weights * 6 * Fraction(2) ** 125 / Fraction(2) ** int(lift) * 4 < limit * Fraction(9, 10)
            # what may count as nothing: below 2^-126, of a largest weight of 2^top
            assert 67 < byte <= 227 and (byte == 227 or n > 2 ** 14)
            assert -126 + lift - top <= (-94 if n <= 2 ** 25 else (n - 1).bit_length() - 119)
