"""Builds libsparse_prefill.so (HIP, gfx950 only) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsparse_prefill.so")
SOURCES = ("api.hip", "pool.hip", "select.hip", "select_d128.hip", "select_d64.hip", "attn.hip",
           "paged_api.hip", "paged_cache.hip", "paged_attn.hip")
HEADERS = ("attn_parts.hpp", "common.hpp", "overlap.hpp", "paged.hpp", "row_deal.hpp", "score_rows.hpp", "select_impl.hpp", "value_block.hpp", os.path.join("..", "..", "include", "sparse_prefill.h"))

# The attention kernel never produces NaN from finite inputs; telling the compiler so
# removes the NaN-quieting v_max x,x pairs it otherwise puts around every fmaxf.
EXTRA = {"attn.hip": ["-fno-honor-nans"]}

# Packed-FP32 VALU forms are switched off for device code on purpose.
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-Wall", "-Wno-unused-function",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS]
    return any(os.path.getmtime(os.path.normpath(d)) > t for d in deps)


def build_library(force: bool = True, verbose: bool = False) -> str:
    """Compile every HIP source and link the shared library.  Compiles each
    time it is called unless force=False and the library is up to date."""
    if not force and not is_stale():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objs, procs = [], []
    os.makedirs(os.path.join(HERE, "_build"), exist_ok=True)
    for s in SOURCES:
        o = os.path.join(HERE, "_build", s.replace(".hip", ".o"))
        cmd = [hipcc, *FLAGS, *EXTRA.get(s, []), "-c", os.path.join(CSRC, s), "-o", o]
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(o)
    for cmd, pr in procs:
        out, _ = pr.communicate()
        out = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l)
        if pr.returncode != 0:
            raise RuntimeError("hipcc failed: " + " ".join(cmd) + "\n" + out)
        if verbose and out.strip():
            print(out)
    link = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    subprocess.run(link, check=True)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
