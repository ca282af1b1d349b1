"""Compiles the CUDA library in-tree for sm_100a (nvcc cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import tempfile

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libad_b200.so")
SOURCES = ["ad_api.cu", "cache_api.cu", "pool_api.cu", "shared_api.cu"]
HEADERS = ["ad_common.cuh", "gemm_tc.cuh", "gemm_tc_pair.cuh", "gemm_simt.cuh", "gemm_few.cuh", "attention.cuh", "attention_few.cuh", "attention_mma.cuh", "ffn_few.cuh", "sublayer_f32.cuh", "steps.cuh", "accept.cuh", "grid_sync.cuh", "mega.cuh", "kv_cache.cuh", "cache_attention.cuh", "accept_sampled.cuh", "shared_attention.cuh", "block_pool.cuh", "sample.cuh", "cache_checks.h", "op_launch.h"]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS]
    deps.append(os.path.join(os.path.dirname(_HERE), "include", "aggressive_decoding.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Builds libad_b200.so next to this file if it is missing or older than its sources."""
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB + f".{os.getpid()}.tmp"
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC", "-cudart", "shared"]
    if verbose:
        flags += ["-Xptxas", "-v"]
    with tempfile.TemporaryDirectory() as folder:
        objects = [os.path.join(folder, s[:-3] + ".o") for s in SOURCES]
        running = [subprocess.Popen([nvcc, *flags, "-rdc=true", "-c", os.path.join(CSRC, s), "-o", o]) for s, o in zip(SOURCES, objects)]
        codes = [r.wait() for r in running]
        if any(codes):
            raise RuntimeError("compilation failed: " + ", ".join(s for s, c in zip(SOURCES, codes) if c))
        subprocess.run([nvcc, *flags, "-shared", "-rdc=true", "-lcudadevrt", *objects, "-o", tmp], check=True)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
