"""Builds the C-ABI shared library (CUDA, sm_100a) in-tree with nvcc.  No GPU is needed to build."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libtrimkv.so")
SOURCES = ["trimkv_runtime.cu", "gate.cu", "gate_tc.cu", "cache.cu", "select.cu", "select_flat.cu", "select_static.cu", "attention.cu", "prefill_attention.cu", "prefill_attention_tc.cu", "paged_plan.cu", "paged_select.cu", "paged_attention.cu", "paged_attention_warp.cu", "paged_attention_tc.cu", "paged_api.cu", "paged4_append.cu", "paged4_attention.cu", "paged4_attention_tc.cu", "paged4_api.cu", "paged_share.cu", "paged_move.cu", "paged_share_api.cu"]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    raise RuntimeError("nvcc not found")


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu to an object and link libtrimkv.so next to this file.  Returns the library path."""
    nvcc = _nvcc()
    headers = [os.path.join(CSRC, "trimkv_internal.cuh"), os.path.join(CSRC, "async_copy.cuh"), os.path.join(CSRC, "mma_sync.cuh"), os.path.join(CSRC, "paged.cuh"), os.path.join(CSRC, "paged_check.cuh"), os.path.join(CSRC, "paged4.cuh"), os.path.join(CSRC, "paged_tc.cuh"), os.path.join(CSRC, "paged_share.cuh"), os.path.join(CSRC, "paged_bounds.cuh"), os.path.join(CSRC, "tcgen05_attn.cuh"), os.path.join(ROOT, "include", "trimkv.h"), __file__]
    objs = []
    procs = []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(CSRC, src.replace(".cu", ".o"))
        objs.append(o)
        if force or _stale(o, [s] + headers):
            cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", s, "-o", o]
            procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for cmd, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode != 0:
            sys.stderr.write(out)
        if p.returncode != 0:
            raise RuntimeError("nvcc failed: " + " ".join(cmd))
    if force or procs or _stale(LIB, objs):
        cmd = [nvcc, "-shared", "-o", LIB] + objs + ["-gencode", "arch=compute_100a,code=sm_100a"]
        r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        if r.returncode != 0:
            sys.stderr.write(r.stdout)
            raise RuntimeError("link failed: " + " ".join(cmd))
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
