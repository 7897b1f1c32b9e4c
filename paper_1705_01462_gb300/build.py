"""Builds libfgq.so (the FGQ CUDA library) in-tree for sm_103a with nvcc.

Each translation unit is compiled in parallel; the objects are linked into
``paper_1705_01462_gb300/libfgq.so`` against the shared CUDA runtime.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libfgq.so")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")

SOURCES = ["api.cu", "ternarize.cu", "ternarize_threshold.cu", "quantize.cu", "gemm_simt.cu", "gemm_simt_g4.cu",
           "gemm_simt_g8.cu", "gemm_simt_g32.cu", "gemm_simt_g128.cu", "gemm_tc.cu", "gemm_tc4.cu", "gemm_fold.cu", "gemm_dense.cu",
           "gemm_few.cu", "gemv.cu", "elementwise.cu", "kv_cache.cu", "kv_attention.cu", "kv_prompt.cu", "kv_attention_d64.cu",
           "kv_attention_d128.cu", "kv_attention_d256.cu", "linear_w8a8.cu", "gemm_w8a8.cu",
           "rope.cu", "add_norm.cu", "linear_w4.cu", "gemm_w4.cu", "gemm_w4_experts.cu", "w4_rows_bf16.cu", "w4_rows_f16.cu", "w4_rows_f32.cu", "moe_w4.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-fno-strict-aliasing",
              "--expt-relaxed-constexpr", "-I" + INCLUDE]


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the FGQ CUDA library cannot be built")


def _deps_mtime() -> float:
    files = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(INCLUDE, f) for f in os.listdir(INCLUDE)] + [__file__]
    return max(os.path.getmtime(f) for f in files)


def up_to_date() -> bool:
    return os.path.exists(LIB) and os.path.getmtime(LIB) >= _deps_mtime()


def build(force: bool = False, verbose: bool = False, extra_flags=None, lib_path: str = LIB,
          build_dir: str = BUILD) -> str:
    """Compile and link the library; extra_flags go to every nvcc compile (e.g. -D options
    for a differently configured copy written to lib_path)."""
    if not force and lib_path == LIB and not extra_flags and up_to_date():
        return LIB
    os.makedirs(build_dir, exist_ok=True)
    cc = nvcc()
    flags = NVCC_FLAGS + list(extra_flags or [])

    def compile_one(src):
        obj = os.path.join(build_dir, src.replace(".cu", ".o"))
        cmd = [cc] + ARCH + flags + ["-c", os.path.join(CSRC, src), "-o", obj]
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError(f"nvcc failed for {src}:\n{' '.join(cmd)}\n{res.stdout}\n{res.stderr}")
        if verbose and (res.stdout or res.stderr):
            sys.stderr.write(res.stdout + res.stderr)
        return obj

    with cf.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = lib_path + f".tmp{os.getpid()}"
    cmd = [cc] + ARCH + ["-shared", "-cudart", "shared", "-o", tmp] + objs
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed:\n{' '.join(cmd)}\n{res.stdout}\n{res.stderr}")
    os.replace(tmp, lib_path)
    return lib_path


if __name__ == "__main__":
    v = "-v" in sys.argv
    print(build(force="--force" in sys.argv, verbose=v,
                extra_flags=["-Xptxas", "-v"] if "--ptxas-v" in sys.argv else None))
