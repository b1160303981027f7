"""Builds libmmee.so in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import shutil
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmmee.so")
SOURCES = ["mmee_plan.cu", "mmee_search.cu", "mmee_views.cu", "mmee_api.cu", "mmee_workspace.cu", "mmee_alu_peak.cu", "mmee_static.cu", "mmee_prune.cu",
           "mmee_chain.cu", "mmee_attention.cu", "mmee_attention_token.cu", "mmee_attention_grad.cu", "mmee_ffn.cu", "mmee_ffn_tokens.cu", "mmee_ffn_narrow.cu"]
HEADERS = ["mmee_plan.h", "mmee_search.h", "mmee_workspace.h", "mmee_eval.cuh", "mmee_classes.cuh", "mmee_block.cuh",
           "mmee_chain.h", "mmee_sm100.cuh", "mmee_attention.cuh", "mmee_ffn.cuh", os.path.join("..", "..", "include", "mmee.h")]
NVCC_FLAGS = ["-t", "0", "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
              "-Xcompiler", "-fPIC", "-shared", "--expt-relaxed-constexpr"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: libmmee.so cannot be built")


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    built = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS]
    return any(os.path.getmtime(d) > built for d in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile every CUDA source of the library into one shared object next to this file."""
    if not force and not is_stale():
        return LIB
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [_nvcc()] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + \
          ["-I", os.path.join(HERE, "..", "include"), "-o", tmp] + [os.path.join(CSRC, s) for s in SOURCES]
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
