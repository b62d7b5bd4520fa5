"""Builds libsepllm.so (sm_100a) in-tree with nvcc.  No GPU is needed to build."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libsepllm.so")
SOURCES = ["index.cu", "index_packed.cu", "cache.cu", "attn_fwd.cu", "attn_fwd_pair.cu", "attn_bwd.cu", "rope.cu", "prefix.cu", "cache_quant.cu", "qknorm.cu",
           "api.cu"]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(INCLUDE, "sepllm.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
             "-I", INCLUDE, "-Xcompiler", "-fPIC"] + (["-Xptxas", "-v"] if verbose else [])

    def run(args):
        r = subprocess.run(flags + args, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("nvcc failed:\n" + r.stdout + r.stderr)
        if verbose:
            print(r.stderr)

    # one compiler per source, side by side, then one link
    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor(os.cpu_count()) as pool:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        for job in [pool.submit(run, ["-c", os.path.join(CSRC, s), "-o", o]) for s, o in zip(SOURCES, objects)]:
            job.result()
        run(["-shared", "-o", LIB] + objects)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
