"""Builds the CUDA library in-tree with nvcc for sm_100a (no JIT cache, no fallback)."""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import sys
import time

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libgn_b200.so")
SOURCES = ["gn_context.cu", "gemm_ffma.cu", "gemm_tf32.cu", "gemm_f16x3.cu", "gemm_thin.cu", "half_copy.cu", "small_net.cu", "vector_ops.cu",
           "layer_norm.cu", "dropout.cu", "gated_ffn.cu",
           "gemm_pair16.cu", "gemm_narrow16.cu", "ffn_dot.cu", "ffn_small.cu",
           "route.cu", "experts.cu", "expert_rows.cu", "gemm_group16.cu", "gemm_group32.cu", "gemm_group_fma.cu",
           "weight4.cu", "weight4_f32.cu", "weight4_bf16.cu", "weight4_f16.cu"]
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
    source and headers are older than its object is taken over, if it was compiled by the same command, unless `force`."""
    if not force and not is_stale():
        return LIB
    nvcc = os.environ.get("NVCC", "nvcc")
    # GN_NVTX=1: named ranges around the phases of the path for timeline tools (header-only NVTX, off by default)
    extra = ["-DGN_NVTX"] if os.environ.get("GN_NVTX") == "1" else []
    compiler = [nvcc] + [f for f in FLAGS if f != "-shared"] + extra
    out_dir = os.path.join(HERE, "_build")
    os.makedirs(out_dir, exist_ok=True)
    objects = [os.path.join(out_dir, s + ".o") for s in SOURCES]
    command = os.path.join(out_dir, "command")           # that the objects were compiled by
    if not os.path.exists(command) or open(command).read() != "\n".join(compiler):
        for obj in objects:
            if os.path.exists(obj):
                os.remove(obj)
        with open(command, "w") as f:
            f.write("\n".join(compiler))
    newest = max(os.path.getmtime(p) for p in _deps() if not p.endswith(".cu"))

    def compile_one(source, obj):
        if not force and os.path.exists(obj) and os.path.getmtime(obj) > max(newest, os.path.getmtime(os.path.join(CSRC, source))):
            return
        _make(compiler + (["-Xptxas", "-v"] if verbose else []), ["-c", source], obj, verbose)

    begin = time.time()
    with concurrent.futures.ThreadPoolExecutor(os.cpu_count() or 1) as pool:
        list(pool.map(compile_one, SOURCES, objects))
    _make([nvcc] + FLAGS, objects, LIB, verbose, begin)
    return LIB


def _make(command, args, out, verbose, begin=None):
    """Run `command -o out args`.  `out` is there whole or not at all, and as old as what was read for it may be: an edit made meanwhile is newer."""
    begin = begin or time.time()
    part = f"{out}.{os.getpid()}.part"
    try:
        res = subprocess.run(command + ["-o", part] + args, cwd=CSRC, capture_output=True, text=True)
        if verbose:
            sys.stderr.write(res.stderr)
        if res.returncode != 0:
            raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
        os.utime(part, (begin, begin))
        os.replace(part, out)
    finally:
        if os.path.exists(part):
            os.remove(part)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
