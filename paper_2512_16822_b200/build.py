"""Build libmepic.so (host store + sm_100a kernels) in-tree with nvcc.

``python -m paper_2512_16822_b200.build`` or ``build_library()``.  The shared
library lands next to this file so that it travels with the source tree; it is
rebuilt only when a source or header is newer than it.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB_PATH = os.path.join(HERE, "libmepic.so")

SOURCES = ["mepic_store.cpp", "mepic_tensor_map.cu", "mepic_decode.cu", "mepic_decode_fp8.cu", "mepic_decode_grouped.cu", "mepic_plan.cpp",
           "mepic_prefill.cu", "mepic_step.cu", "mepic_tree.cu", "mepic_beam.cu", "mepic_attn_beam.cu"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the MEPIC library needs the CUDA toolkit to build")


def _stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    built = os.path.getmtime(LIB_PATH)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(INCLUDE, f) for f in os.listdir(INCLUDE)]
    return any(os.path.getmtime(d) > built for d in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile for sm_100a; returns the path of the shared library."""
    if not force and not _stale():
        return LIB_PATH
    srcs = [os.path.join(CSRC, s) for s in SOURCES if os.path.exists(os.path.join(CSRC, s))]
    cmd = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-shared", "-Xcompiler", "-fPIC", "-cudart", "static",
           "-I", INCLUDE, "-I", CSRC, "-o", LIB_PATH + ".tmp"]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += os.environ.get("MEPIC_NVCC_FLAGS", "").split()      # extra flags for experiments (e.g. -DMEPIC_DECODE_STAGES=2)
    cmd += srcs      # libcuda is NOT linked: the library must load on a machine without a driver
    proc = subprocess.run(cmd, capture_output=True, text=True)
    if proc.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + " ".join(cmd) + "\n" + proc.stdout + proc.stderr)
    if verbose:
        print(proc.stdout + proc.stderr)
    os.replace(LIB_PATH + ".tmp", LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
