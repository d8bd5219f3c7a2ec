"""Builds the HIP libraries in-tree (gfx950 only): paper_2012_15198_amd/libcxmix.so, the mixing library, and libcxlm.so, the
language-model operators."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libcxmix.so")
CSRC = os.path.join(HERE, "csrc")
SOURCES = [os.path.join(CSRC, f) for f in ("cx_host.cpp", "cx_hbm.cpp", "cx_api_gossip.hip", "cx_api_hier.hip",
                                           "cx_api_pushsum.hip", "cx_api_fused.hip", "cx_api_hiersgd.hip",
                                           "cx_api_bf16.hip", "cx_api_f16.hip", "cx_api_hier16.hip",
                                           "cx_api_noalloc.hip", "cx_api_fused16.hip", "cx_api_pushsum16.hip")]
HEADERS = [os.path.join(ROOT, "include", "cx_mix.h")] + [os.path.join(CSRC, h) for h in (
    "cx_columns.hpp", "cx_schedule.hpp", "cx_tile.hpp", "cx_ops.hpp", "cx_ops16.hpp", "cx_kernels.hpp", "cx_launch.hpp")]
LM_LIB = os.path.join(HERE, "libcxlm.so")
LM_CSRC = os.path.join(CSRC, "lm")
LM_SOURCES = [os.path.join(LM_CSRC, f) for f in ("cx_lm_embed.hip", "cx_lm_scan.hip", "cx_lm_scores.hip", "cx_lm_distill.hip",
                                                 "cx_lm_norm.hip", "cx_lm_conv.hip", "cx_lm_select.hip", "cx_lm_select_grad.hip")]
LM_HEADERS = [os.path.join(ROOT, "include", h) for h in ("cx_lm.h", "cx_mix.h")] + [os.path.join(LM_CSRC, h) for h in (
    "lm_common.hpp", "lm_vocab.hpp", "lm_block.hpp", "lm_select.hpp")]
OBJDIR = os.path.join(HERE, "_build")

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC",
    "-ffp-contract=off",                      # the fp32 formulas are specified without FMA
    "-fno-fast-math",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",   # no packed fp32 math
    "-Wall", "-Wextra", "-Wno-unused-parameter",
]


def stale(lib: str = LIB, files=None) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    return any(os.path.getmtime(p) > t for p in files or SOURCES + HEADERS)


def build_library(force: bool = True, verbose: bool = False) -> str:
    """Compile every HIP/C++ source of the libraries for gfx950 (cross-compiles without a GPU).  The mixing library's path."""
    wanted = [(lib, sources) for lib, sources, headers in ((LIB, SOURCES, HEADERS), (LM_LIB, LM_SOURCES, LM_HEADERS))
              if force or stale(lib, sources + headers)]
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    os.makedirs(OBJDIR, exist_ok=True)
    obj_of = lambda src: os.path.join(OBJDIR, os.path.basename(src) + ".o")

    def compile_one(src):
        cmd = [hipcc, *HIPCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-c", src, "-o", obj_of(src)]
        if verbose:
            print(" ".join(cmd), file=sys.stderr)
        subprocess.check_call(cmd)

    # one translation unit per entry point: compile them side by side, then link
    todo = [src for _, sources in wanted for src in sources]
    if todo:
        with ThreadPoolExecutor(max_workers=min(len(todo), int(os.environ.get("MAX_JOBS", "8")))) as pool:
            list(pool.map(compile_one, todo))
    for lib, sources in wanted:
        link = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *map(obj_of, sources), "-o", lib]
        if verbose:
            print(" ".join(link), file=sys.stderr)
        subprocess.check_call(link)
    return LIB


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
