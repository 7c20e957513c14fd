"""Builds librlkv.so in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "librlkv.so")
SOURCES = ["rlkv_api.cu", "rlkv_paged.cu", "rlkv_prompt.cu", "rlkv_paged_chunks.cu", "append_kernel.cu", "rotary_kernel.cu",
           "norm_rotary.cu", "chunk_rows.cu", "decode_kernel.cu", "chunk_attention.cu", "prompt_forward.cu", "prompt_backward.cu", "probe_kernel.cu"]
HEADERS = ["rlkv_internal.cuh", "rlkv_host.cuh", "rlkv_paged.cuh", "rlkv_prompt.cuh", "rlkv_chunk.cuh", "rotary.cuh", "tcgen05.cuh", os.path.join("..", "..", "include", "rlkv.h")]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC"]
# Fast-math (approximate exp2 and division, flush-to-zero) is wanted in the decode kernel's softmax and
# nowhere else: the append kernel's quantiser and the host arithmetic keep IEEE behaviour.
EXTRA_FLAGS = {"decode_kernel.cu": ["--use_fast_math"]}
OBJ_DIR = os.path.join(PKG, "_build")


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    built = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS] + [os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > built for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile the library if it is missing or older than its sources; returns its path."""
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "nvcc")
    os.makedirs(OBJ_DIR, exist_ok=True)
    objs, procs = [], []
    for src in SOURCES:                       # one object per source, compiled side by side
        obj = os.path.join(OBJ_DIR, src.replace(".cu", ".o"))
        cmd = [nvcc] + NVCC_FLAGS + EXTRA_FLAGS.get(src, []) + (["-Xptxas", "-v"] if verbose else []) + \
              ["-c", os.path.join(CSRC, src), "-o", obj]
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    failed = False
    for src, proc in procs:
        out, _ = proc.communicate()
        if verbose or proc.returncode != 0:
            sys.stderr.write(out)
        failed = failed or proc.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed building librlkv.so")
    res = subprocess.run([nvcc, "-shared", "-gencode", "arch=compute_100a,code=sm_100a"] + objs + ["-o", LIB],
                         capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("nvcc failed linking librlkv.so")
    return LIB


if __name__ == "__main__":
    build(force=True, verbose="-v" in sys.argv)
    print(LIB)
