"""Build libaecct.so in-tree with nvcc for sm_103a (GB300).

The CUDA sources are compiled in parallel (one nvcc per translation unit) and linked into
paper_2410_05911_gb300/_build/libaecct.so.  The decoder's translation unit is built with
--fmad=false so that no multiply-add is contracted behind the explicit fp32 operation order.
"""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT_DIR = os.path.join(HERE, "_build")
LIB_PATH = os.path.join(OUT_DIR, "libaecct.so")
SOURCES = ["api.cu", "decoder_kernel.cu", "decoder_kernel_gelu.cu", "decoder_kernel_fp.cu", "decoder_kernel_fp_gelu.cu",
           "decoder_kernel_cap.cu", "decoder_kernel_cap_fp.cu", "selftest.cu", "aap.cu", "spe.cu",
           "norm.cu", "clip.cu", "linear.cu", "linear_grad.cu", "linear_wgrad.cu",
           "linear_stage.cu"]
HEADERS = ["aecct_internal.h", "sm103_ptx.cuh", "rowtypes.cuh", "linear_gemm.cuh", "decoder_kernel.cuh", os.path.join("..", "..", "include", "aecct.h")]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ARCH + ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "--fmad=false",
                     "-Xcompiler", "-fno-strict-aliasing"]


def nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS] + [os.path.abspath(__file__)]
    return any(os.path.getmtime(p) > t for p in deps if os.path.exists(p))


def build(force: bool = False, verbose_ptxas: bool = False) -> str:
    """Compile (if needed) and return the path of libaecct.so."""
    if not force and not _stale():
        return LIB_PATH
    os.makedirs(OUT_DIR, exist_ok=True)
    procs = []
    objs = []
    for src in SOURCES:
        obj = os.path.join(OUT_DIR, os.path.splitext(src)[0] + ".o")
        objs.append(obj)
        cmd = [nvcc(), *NVCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose_ptxas:
            cmd.insert(1, "-Xptxas=-v")
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = []
    for src, pr in procs:
        out, _ = pr.communicate()
        if out and (verbose_ptxas or pr.returncode):
            sys.stderr.write(out)
        if pr.returncode:
            failed.append(src)
    if failed:
        raise RuntimeError(f"nvcc failed for {failed}")
    tmp = LIB_PATH + f".tmp{os.getpid()}"
    subprocess.check_call([nvcc(), *ARCH, "-shared", "-o", tmp, *objs])
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose_ptxas="-v" in sys.argv))
