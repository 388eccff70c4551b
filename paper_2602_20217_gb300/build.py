"""Build libknapspec.so in-tree: one nvcc per translation unit (in parallel),
sm_103a only, then a shared-library link against the CUDA runtime."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libknapspec.so")
SOURCES = ["chain.cu", "gemv.cu", "attn.cu", "select.cu", "sample.cu", "dp.cu", "model.cu", "wide.cu", "wide_attn.cu",
           "kv8.cu", "kv8_attn.cu", "kv8_tc.cu", "kv8_shared.cu", "kv8_weights.cu",
           "kv8_weights_tc.cu", "kv8_evict.cu", "logprob.cu"]
HEADERS = ["common.cuh", "internal.h", "tma.cuh", "umma.cuh", "kv8.h", "kv8.cuh", "kv8_plan.cuh"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-O2"]


def nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is needed to build libknapspec")


def _deps_mtime() -> float:
    files = [os.path.join(CSRC, h) for h in HEADERS]
    files.append(os.path.join(ROOT, "include", "knapspec.h"))
    files.append(os.path.abspath(__file__))
    return max(os.path.getmtime(f) for f in files)


def build(verbose: bool = False, force: bool = False) -> str:
    """Compile (if stale) and return the path of libknapspec.so."""
    os.makedirs(BUILD, exist_ok=True)
    nv = nvcc()
    dep_t = _deps_mtime()
    jobs = []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(BUILD, src.replace(".cu", ".o"))
        stale = force or not os.path.exists(o) or os.path.getmtime(o) < max(os.path.getmtime(s), dep_t)
        jobs.append((s, o, stale))

    def compile_one(job):
        s, o, stale = job
        if not stale:
            return None
        cmd = [nv, *ARCH, *FLAGS, "-I", os.path.join(ROOT, "include"), "-c", s, "-o", o]
        if verbose:
            print(" ".join(cmd), file=sys.stderr)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            return f"{os.path.basename(s)}:\n{r.stdout}\n{r.stderr}"
        return None

    with ThreadPoolExecutor(max_workers=len(jobs)) as ex:
        errors = [e for e in ex.map(compile_one, jobs) if e]
    if errors:
        raise RuntimeError("nvcc failed:\n" + "\n".join(errors))
    objs = [o for _, o, _ in jobs]
    if force or not os.path.exists(LIB) or os.path.getmtime(LIB) < max(os.path.getmtime(o) for o in objs):
        tmp = LIB + ".tmp"
        cmd = [nv, *ARCH, "-shared", "-o", tmp, *objs, "-lcudart"]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
        os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True, force="--force" in sys.argv))
