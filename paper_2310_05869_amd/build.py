"""Builds libhyperattn.so (gfx950) from csrc/ with hipcc, in-tree.

    python -m paper_2310_05869_amd.build

hipcc cross-compiles without a GPU.  Objects go to csrc/_build/ (ignored by
git); the shared library lands next to this file, where the binding loads it.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(CSRC, "_build")
LIB = os.path.join(HERE, "libhyperattn.so")

SOURCES = ["api.hip", "lsh_hash.hip", "lsh_hash_mfma.hip", "seg_sort.hip", "stage_kernels.hip", "attn_mfma.hip", "attn_f32.hip",
           "calib.hip", "attn_bwd_mfma.hip", "attn_bwd_f32.hip", "bwd_kernels.hip", "alg2_kernels.hip", "alg2_mfma.hip",
           "page_plan.hip", "cache4_rows.hip", "cache4_attn.hip", "cache_api.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed-fp32 instructions stay off: some of their forms have returned wrong results on this hardware
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _compile(src: str, extra: list[str]) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *FLAGS, *extra, "-c", os.path.join(CSRC, src), "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in res.stderr.splitlines() if "packed-fp32-ops" not in l)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{err}")
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def build_library(extra_flags: list[str] | None = None, jobs: int = 6) -> str:
    os.makedirs(BUILD, exist_ok=True)
    extra = list(extra_flags or [])
    with ThreadPoolExecutor(max_workers=jobs) as ex:
        objs = list(ex.map(lambda s: _compile(s, extra), SOURCES))
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("link failed:\n" + res.stderr)
    return LIB


if __name__ == "__main__":
    print(build_library(sys.argv[1:]))
