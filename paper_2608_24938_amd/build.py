"""Build libexfold.so (all HIP sources, gfx950) in-tree.

    python -m paper_2608_24938_amd.build        # or build() from Python

Every source is compiled with hipcc for gfx950 only; packed fp32 VALU
instructions are disabled (the compiler would otherwise form them from plain
float code).  The library lands next to this file.
"""

from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(PKG, "_build")
LIB_PATH = os.path.join(PKG, "libexfold.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"
FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-Wall",
    "-Wno-unused-function", "-Wno-unused-variable",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # keep per-thread address arrays in registers (the pass would move them to LDS)
    "-mllvm", "-disable-promote-alloca-to-lds",
    f"-I{INCLUDE}", f"-I{CSRC}",
]
SOURCES = ["exfold_api.hip", "k_route.hip", "k_score.hip", "k_permute.hip", "k_gemm.hip", "k_linear.hip",
           "k_calib.hip", "k_diag.hip"]


def _run(cmd):
    res = subprocess.run(cmd, capture_output=True, text=True)
    # hipcc's host pass does not know the packed-fp32 feature and says so; that is harmless
    noise = "'-packed-fp32-ops' is not a recognized feature"
    err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
    if res.returncode != 0:
        raise RuntimeError(f"command failed ({res.returncode}): {' '.join(cmd)}\n{err}")
    return err


def build(verbose: bool = False, jobs: int = 8) -> str:
    """Compile every HIP source for gfx950 and link libexfold.so; returns its path."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    objs = []
    cmds = []
    for src in SOURCES:
        obj = os.path.join(BUILD_DIR, src.replace(".hip", ".o"))
        objs.append(obj)
        cmds.append([HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj])
    with ThreadPoolExecutor(max_workers=max(1, min(jobs, len(cmds)))) as ex:
        for cmd, warn in zip(cmds, ex.map(_run, cmds)):
            if verbose and warn.strip():
                print(warn, file=sys.stderr)
    tmp = LIB_PATH + ".tmp"
    _run([HIPCC, *FLAGS, "-shared", "-o", tmp, *objs])
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
