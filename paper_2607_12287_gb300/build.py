"""Builds the CUDA library ``_build/libivit.so`` for sm_103a with nvcc.

The translation units compile in parallel; the shared object links the CUDA
runtime statically, so loading it needs no GPU and no driver library.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OUT_DIR = os.path.join(HERE, "_build")
LIB = os.path.join(OUT_DIR, "libivit.so")
SOURCES = ["gemm.cu", "gemm_pair.cu", "ops.cu", "attention.cu", "attention_rows.cu", "persistent.cu", "stream.cu", "engine.cu", "noalloc.cu",
           "action.cu", "step_plan.cu", "rope.cu", "tree_attention.cu", "tree_attention_tc.cu", "kv_write.cu",
           "kv_quantise.cu", "tree_attention_quantised.cu", "tree_attention_quantised_fp16.cu", "tree_attention_quantised_tc.cu",
           "tree_verify.cu"]
HEADERS = ["ptx.cuh", "internal.h", "select.cuh", "attention.cuh", "gelu.cuh", "backbone.cuh", "tree_attention.cuh", "tree_join.cuh", "quantised.cuh",
           "tree_attention_quantised.cuh"]
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include")]


def _mtime(p: str) -> float:
    return os.path.getmtime(p) if os.path.exists(p) else 0.0


def build(force: bool = False, verbose: bool = False) -> str:
    os.makedirs(OUT_DIR, exist_ok=True)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS] + [os.path.join(ROOT, "include", "ivit.h")]
    if not force and _mtime(LIB) > max(_mtime(d) for d in deps):
        return LIB

    def compile_one(src: str) -> str:
        obj = os.path.join(OUT_DIR, src.replace(".cu", ".o"))
        cmd = [NVCC, *ARCH, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
        if verbose:
            sys.stderr.write(r.stderr)
        return obj

    with ThreadPoolExecutor(len(SOURCES)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = LIB + f".tmp{os.getpid()}"
    r = subprocess.run([NVCC, *ARCH, "-shared", "-o", tmp, *objs], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
