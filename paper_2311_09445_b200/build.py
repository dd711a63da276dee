"""Builds libpearl_prb.so (the CUDA kernels + C ABI) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libpearl_prb.so")
LIB_CHECKED = os.path.join(HERE, "libpearl_prb_checked.so")     # every index checked against its extent (-DPEARL_CHECKED)
SOURCES = ["prb_host.cu", "prb_insert.cu", "prb_sample.cu", "prb_sample_short.cu", "prb_step.cu", "prb_tree.cu", "prb_update.cu", "prb_update_wide.cu",
           "rows_host.cu", "rows_route.cu", "rows_sort.cu", "rows_copy.cu", "rows_beam.cu",
           "layer_host.cu", "layer_norm.cu", "layer_dropout.cu", "layer_experts.cu"]

NVCC_FLAGS = [
    "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
    "--extended-lambda",
    # bit-exact contract with the CPU restatement: no contraction, no flush-to-zero, IEEE div/sqrt
    "-fmad=false", "-ftz=false", "-prec-div=true", "-prec-sqrt=true",
    "-Xcompiler", "-fPIC", "-shared",
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def needs_build(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    deps += [os.path.join(os.path.dirname(HERE), "include", h) for h in ("pearl_prb.h", "pearl_rows.h", "pearl_layers.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False, checked: bool = False) -> str:
    """Builds the library (checked=True: the bounds-checked variant, used through PEARL_PRB_LIB)."""
    lib = LIB_CHECKED if checked else LIB
    if not force and not needs_build(lib):
        return lib
    tmp = lib + ".%d.tmp" % os.getpid()
    cmd = [_nvcc()] + NVCC_FLAGS + (["-DPEARL_CHECKED"] if checked else []) + (["-Xptxas", "-v"] if verbose else []) + \
          ["-o", tmp] + [os.path.join(CSRC, s) for s in SOURCES]
    subprocess.check_call(cmd)
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, checked="--checked" in sys.argv))
