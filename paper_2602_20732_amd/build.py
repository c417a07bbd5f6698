"""Builds ``libchess.so`` (the HIP kernels and their C ABI) in-tree with hipcc for gfx950."""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libchess.so")
SOURCES = ["api.hip", "summarize.hip", "select.hip", "decode.hip", "step.hip", "shared.hip", "trigger.hip", "pages.hip",
           "quant_store.hip", "quant_summarize.hip", "quant_decode.hip", "rotate.hip", "attend.hip", "verify.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared", "-fno-gpu-rdc",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         # the first arguments of a kernel (as far as they are pointers and numbers, not structs) are in registers when it starts:
         # its first loads need no argument fetch (32 layers of a reuse step 236.5 -> 231.8 us)
         "-mllvm", "-amdgpu-kernarg-preload-count=16", "-Wall", "-Wno-unused-command-line-argument"]


def build(verbose: bool = False) -> str:
    """Compile every source, every time (cross-compiles without a GPU)."""
    cmd = ["hipcc", *FLAGS, *[os.path.join(CSRC, s) for s in SOURCES], "-o", LIB]
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + err)
    if verbose and err.strip():
        print(err)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
