"""Builds libfalqon.so (the CUDA kernels and their C ABI) in-tree for sm_100a with nvcc."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libfalqon.so")
SOURCES = ["api.cu", "quantize.cu", "gemm_fp8.cu", "gemm_fp8_fused.cu", "gemm_db.cu", "update_a.cu", "proxy_update.cu", "proxy_update_static.cu", "chain_ops.cu", "chain_quant.cu", "checkpoint.cu", "block_norm.cu", "preference.cu", "block_quant.cu", "block_product.cu", "block_linear.cu", "orthogonalize.cu", "ortho_thin.cu", "merge_exact.cu", "svd_init.cu", "tensor_ceiling.cu"]
HEADERS = ["internal.h", "ptx.cuh", "gemm_common.cuh", "convert_tile.cuh", "chain_math.cuh", "grid_sync.cuh", "mx8.cuh", "block_linear.h", "ortho_thin.h", "tile_walk.cuh", os.path.join("..", "..", "include", "falqon.h"),
           os.path.join("..", "..", "include", "falqon_chain.h"),
           os.path.join("..", "..", "include", "falqon_train.h"),
           os.path.join("..", "..", "include", "falqon_dense.h")]
NVCC_FLAGS = ["-std=c++17", "-O3", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC", "-Xptxas", "-v", "-Xptxas", "-dlcm=cg"]


def _newest(paths):
    return max(os.path.getmtime(p) for p in paths)


def build(force: bool = False, verbose: bool = False) -> str:
    srcs = [os.path.join(CSRC, s) for s in SOURCES]
    deps = srcs + [os.path.join(CSRC, h) for h in HEADERS] + [os.path.abspath(__file__)]
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= _newest(deps):
        return LIB
    objdir = os.path.join(HERE, "build")
    os.makedirs(objdir, exist_ok=True)

    def compile_one(src):
        obj = os.path.join(objdir, os.path.basename(src) + ".o")
        res = subprocess.run(["nvcc", *NVCC_FLAGS, "-c", src, "-o", obj], capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError(f"nvcc failed for {src}:\n{res.stdout}\n{res.stderr}")
        return obj, res.stderr

    with ThreadPoolExecutor(max_workers=4) as pool:
        results = list(pool.map(compile_one, srcs))
    if verbose:
        for _, log in results:
            sys.stderr.write(log)
    objs = [o for o, _ in results]
    res = subprocess.run(["nvcc", "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-o", LIB, *objs],
                         capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed:\n{res.stdout}\n{res.stderr}")
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
