"""Build libwici.so (HIP C++ for gfx950) in-tree with hipcc.

    python -m paper_2608_24204_amd.build [-v]

Each source is compiled to an object in parallel, then linked into
paper_2608_24204_amd/libwici.so.  Always rebuilds.
"""

from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OUT = os.path.join(PKG, "libwici.so")
BUILD = os.path.join(PKG, "_build")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

SOURCES = ["gemv.hip", "misc.hip", "attention.hip", "gemm.hip", "batch.hip", "kv8.hip", "kv8_attn.hip",
           "kv4.hip", "kv4_attn.hip", "beam.hip",
           "model.cpp", "ops.cpp", "quant.cpp", "cache.cpp", "noalloc.cpp"]

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Wall", "-Wno-unused-function", "-Wno-unused-variable",
    # packed fp32 instructions are not used on this target
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


# Per-source flags.  The attention sources: matrix-core results in ordinary vector
# registers (not the accumulation registers), so the output rows that the softmax
# rescales are not copied between the two register files on every key block.
_VGPR_RESULTS = ["-mllvm", "-amdgpu-mfma-vgpr-form"]
EXTRA = {"attention.hip": _VGPR_RESULTS, "kv8_attn.hip": _VGPR_RESULTS, "kv4_attn.hip": _VGPR_RESULTS}


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                    if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"command failed: {' '.join(cmd)}\n{out}")
    if verbose and out.strip():
        print(out)


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    objs = []
    cmds = []
    for src in SOURCES:
        obj = os.path.join(BUILD, src + ".o")
        lang = ["-x", "hip"]
        cmds.append([HIPCC, *lang, *FLAGS, *EXTRA.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj])
        objs.append(obj)
    jobs = min(len(cmds), max(1, min(16, os.cpu_count() or 1)))
    with ThreadPoolExecutor(jobs) as ex:
        list(ex.map(lambda c: _run(c, verbose), cmds))
    tmp = OUT + ".tmp"
    _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-pthread", *objs, "-o", tmp], verbose)
    os.replace(tmp, OUT)
    return OUT


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv[1:]))
