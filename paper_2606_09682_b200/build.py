"""Builds ``libamk.so`` (the C-ABI library of include/amk.h) for sm_100a with nvcc, in-tree."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libamk.so")
SOURCES = ["amk_host.cu", "amk_kernel.cu", "amk_kernel_trace.cu", "amk_pack.cu", "amk_static.cu",
           "amk_attn.cu", "amk_logprobs.cu", "amk_compact.cu",
           "amk_rope.cu", "amk_evict.cu", "amk_verify.cu"]
HEADERS = ["amk_layout.h", "amk_internal.h", "amk_ptx.cuh", "amk_kernel_impl.cuh", "amk_op_util.h",
           "amk_op_launch.h", "amk_attn.cuh", "amk_attn_weights.cuh", "amk_weights_units.h", "amk_tc.cuh",
           os.path.join(ROOT, "include", "amk.h")]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + [h if os.path.isabs(h) else os.path.join(CSRC, h) for h in HEADERS]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17", "--threads", "4",
           "-Xcompiler", "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-o", LIB] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError("nvcc failed")
    if verbose:
        sys.stderr.write(r.stderr)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
