"""Build libipdv.so (gfx950) in-tree with hipcc.

    python -m paper_2609_36546_amd.build          # or build() from Python

Every HIP source is compiled for gfx950 only, with packed-fp32 instruction
selection disabled, and linked into paper_2609_36546_amd/libipdv.so.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
OUT = os.path.join(HERE, "libipdv.so")
BUILD_DIR = os.path.join(HERE, "_build")
SOURCES = ["verify_attn.hip", "lmhead.hip", "accept_scan.hip", "kl.hip", "rope.hip", "kv_q8.hip",
           "attn_q8.hip", "sample_logits.hip", "attn_masked.hip", "attn_mass.hip", "evict.hip", "drafts.hip",
           "abi.cpp"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "-x", "hip", "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function", "-I", INCLUDE, "-I", CSRC,
]
# Per-source code generation flags.  The attention kernels keep their MFMA
# accumulators in arch VGPRs (they rescale them with VALU ops);
# the LM-head GEMM needs AGPRs for its 256-register accumulator tile.
EXTRA = {src: ["-mllvm", "-amdgpu-mfma-vgpr-form"]
         for src in ("verify_attn.hip", "attn_q8.hip", "attn_masked.hip", "attn_mass.hip")}


def _run(cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    # the host pass does not know the packed-fp32 feature and says so; harmless
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"{' '.join(cmd)}\n{err}")
    return err


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD_DIR, exist_ok=True)

    def compile_one(src):
        obj = os.path.join(BUILD_DIR, os.path.splitext(src)[0] + ".o")
        msg = _run([HIPCC, *FLAGS, *EXTRA.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj])
        if verbose and msg.strip():
            print(msg, file=sys.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = OUT + ".tmp"
    _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp])
    os.replace(tmp, OUT)
    return OUT


if __name__ == "__main__":
    print(build(verbose=True))
