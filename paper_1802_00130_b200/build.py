"""Builds the CUDA library in-tree with nvcc for sm_100a (no JIT cache, no fallback)."""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libgn_b200.so")
SOURCES = ["gn_context.cu", "gemm_ffma.cu", "gemm_tf32.cu", "gemm_f16x3.cu", "gemm_thin.cu", "half_copy.cu", "small_net.cu", "vector_ops.cu",
           "layer_norm.cu", "dropout.cu", "gated_ffn.cu",
           "gemm_pair16.cu", "gemm_narrow16.cu", "ffn_dot.cu", "ffn_small.cu"]
FLAGS = ["-shared", "-Xcompiler", "-fPIC", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
         "-O3", "-std=c++17"]


def _deps():
    out = [os.path.join(CSRC, s) for s in SOURCES]
    out += [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".h") or f.endswith(".cuh")]
    out.append(os.path.join(os.path.dirname(HERE), "include", "gn.h"))
    return out


def is_stale():
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(p) > t for p in _deps())


def build(force=False, verbose=False):
    """Compile libgn_b200.so next to this file; returns its path.  Each source becomes an object in _build/, several at a time; one whose
    source and headers are older than its object is taken over unless `force`."""
    if not force and not is_stale():
        return LIB
    nvcc = os.environ.get("NVCC", "nvcc")
    # GN_NVTX=1: named ranges around the phases of the path for timeline tools (header-only NVTX, off by default)
    extra = ["-DGN_NVTX"] if os.environ.get("GN_NVTX") == "1" else []
    out_dir = os.path.join(HERE, "_build")
    os.makedirs(out_dir, exist_ok=True)
    newest = max(os.path.getmtime(p) for p in _deps() if not p.endswith(".cu"))

    def compile_one(source):
        src, obj = os.path.join(CSRC, source), os.path.join(out_dir, source + ".o")
        if not force and not extra and os.path.exists(obj) and os.path.getmtime(obj) > max(newest, os.path.getmtime(src)):
            return obj
        cmd = [nvcc] + [f for f in FLAGS if f != "-shared"] + extra + (["-Xptxas", "-v"] if verbose else []) + ["-c", "-o", obj, source]
        _run(cmd, verbose)
        return obj

    with concurrent.futures.ThreadPoolExecutor(os.cpu_count() or 1) as pool:
        objects = list(pool.map(compile_one, SOURCES))
    _run([nvcc] + FLAGS + ["-o", LIB] + objects, verbose)
    return LIB


def _run(cmd, verbose):
    res = subprocess.run(cmd, cwd=CSRC, capture_output=True, text=True)
    if verbose:
        sys.stderr.write(res.stderr)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
