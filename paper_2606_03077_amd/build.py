"""Builds liblibra.so (HIP for gfx950) in-tree with hipcc.

    python -m paper_2606_03077_amd.build          # compile + link
    LIBRA_SAVE_TEMPS=1 python -m paper_2606_03077_amd.build   # keep the gfx950 assembly

Every source is compiled on each call (objects go to ``_build/``); the shared library is
written next to this file, where the binding loads it from.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "liblibra.so")
ARCH = "gfx950"

SOURCES = ["api.cpp", "plan.cpp", "migrate.cpp", "cost_model.cpp", "scheduler.cpp", "kv_layout.hip", "decode.hip", "merge.hip",
           "chunk.hip", "xcd_weights.hip", "scratch.hip", "positions.cpp", "rotary.hip",
           "drafts.cpp", "norm.hip", "kv_map.hip", "tree.hip"]

# Packed-fp32 VALU forms are disabled for all device code (the host pass warns that it
# does not know the feature; that is harmless).  -Wno-inline-asm: the copies to LDS name m0,
# which they set, as clobbered, and each would be warned of.
COMMON = ["-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function", "-Wno-inline-asm", f"-I{INCLUDE}",
          f"-I{CSRC}", f"--offload-arch={ARCH}",
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found (ROCm is required to build libra)")


def _compile(src: str, save_temps: bool) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [hipcc(), *COMMON, "-c", os.path.join(CSRC, src), "-o", obj]
    if save_temps:
        cmd.insert(1, f"-save-temps={'obj'}")
    r = subprocess.run(cmd, capture_output=True, text=True, cwd=BUILD)
    errs = "\n".join(line for line in r.stderr.splitlines()
                     if "packed-fp32-ops" not in line and line.strip())
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{errs}")
    if errs:
        print(errs, file=sys.stderr)
    return obj


def build(verbose: bool = True) -> str:
    os.makedirs(BUILD, exist_ok=True)
    save = os.environ.get("LIBRA_SAVE_TEMPS") == "1"
    with cf.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(lambda s: _compile(s, save), SOURCES))
    tmp = LIB + ".tmp"
    cmd = [hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", "-pthread", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build()
