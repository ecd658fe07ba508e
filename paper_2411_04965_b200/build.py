"""Builds libbitnet_a48.so (sm_100a only) in-tree with nvcc."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libbitnet_a48.so")
SOURCES = ["api.cu", "pack.cu", "quant.cu", "quant_topk.cu", "linear_simple.cu", "gemm_tcgen05.cu", "decode.cu", "decode_sparse.cu", "block.cu", "ffn_gate_first.cu", "attn_lowbit.cu", "decode_trit5.cu", "attn_tcgen05.cu", "paged_cache.cu", "attn_paged.cu", "attn_paged_tc.cu", "quant_fp8.cu", "gemm_fp8.cu", "rows_fp8.cu", "logprobs.cu", "head.cu"]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _newer(target: str, deps: list[str]) -> bool:
    if not os.path.exists(target):
        return False
    t = os.path.getmtime(target)
    return all(os.path.getmtime(d) <= t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    os.makedirs(OBJ, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    headers.append(os.path.join(ROOT, "include", "bitnet_a48.h"))
    extra = ["-Xptxas", "-v"] if verbose else []

    def compile_one(src: str) -> str:
        s = os.path.join(CSRC, src)
        o = os.path.join(OBJ, src.replace(".cu", ".o"))
        if force or not _newer(o, [s] + headers):
            r = subprocess.run(["nvcc", *NVCC_FLAGS, *extra, "-c", s, "-o", o], capture_output=True, text=True)
            if verbose or r.returncode != 0:
                sys.stderr.write(r.stdout + r.stderr)
            if r.returncode != 0:
                raise RuntimeError(f"nvcc failed on {src}")
        return o

    with ThreadPoolExecutor(max_workers=8) as pool:
        objs = list(pool.map(compile_one, SOURCES))
    if force or not _newer(LIB, objs):
        subprocess.run(["nvcc", "-shared", "-gencode", "arch=compute_100a,code=sm_100a", *objs, "-o", LIB], check=True)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
