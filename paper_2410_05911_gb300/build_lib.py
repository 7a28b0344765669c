"""Build libaecct.so in-tree with nvcc for sm_103a (GB300), and its binding to torch's tensors with g++.

The CUDA sources are compiled in parallel (one nvcc per translation unit) and linked into
paper_2410_05911_gb300/_build/libaecct.so; aecct_torch.so beside it links against it and torch.  The decoder's translation unit is built with
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
BINDING_PATH = os.path.join(OUT_DIR, "aecct_torch.so")
BINDING_SOURCE = "torch_binding.cpp"
SOURCES = ["api.cu", "decoder_kernel.cu", "decoder_kernel_gelu.cu", "decoder_kernel_fp.cu", "decoder_kernel_fp_gelu.cu",
           "decoder_kernel_cap.cu", "decoder_kernel_cap_fp.cu", "selftest.cu", "aap.cu", "spe.cu",
           "norm.cu", "clip.cu", "linear.cu", "linear_grad.cu", "linear_wgrad.cu",
           "linear_stage.cu", "linear_few.cu"]
HEADERS = ["aecct_internal.h", "sm103_ptx.cuh", "rowtypes.cuh", "linear_gemm.cuh", "decoder_kernel.cuh", os.path.join("..", "..", "include", "aecct.h")]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ARCH + ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "--fmad=false",
                     "-Xcompiler", "-fno-strict-aliasing"]


def nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _stale() -> bool:
    if not os.path.exists(LIB_PATH) or not os.path.exists(BINDING_PATH):
        return True
    t = min(os.path.getmtime(LIB_PATH), os.path.getmtime(BINDING_PATH))
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS + [BINDING_SOURCE]] + [os.path.abspath(__file__)]
    return any(os.path.getmtime(p) > t for p in deps if os.path.exists(p))


def _binding_command(obj: str):
    """g++ on the binding's source: torch's and Python's headers."""
    import sysconfig

    import torch

    inc = os.path.join(os.path.dirname(torch.__file__), "include")
    dirs = [inc, os.path.join(inc, "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"],
            os.path.join(os.path.dirname(os.path.dirname(nvcc())) or "/usr/local/cuda", "include")]
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-c", os.path.join(CSRC, BINDING_SOURCE), "-o", obj,
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *[a for d in dirs for a in ("-isystem", d)]]


def _link_binding(obj: str) -> None:
    import torch

    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    tmp = BINDING_PATH + f".tmp{os.getpid()}"
    subprocess.check_call(["g++", "-shared", "-o", tmp, obj, "-L" + OUT_DIR, "-l:libaecct.so", "-L" + lib, "-ltorch_python",
                           "-ltorch_cpu", "-ltorch_cuda", "-ltorch", "-lc10", "-lc10_cuda", "-Wl,-rpath,$ORIGIN", "-Wl,-rpath," + lib])
    os.replace(tmp, BINDING_PATH)


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
    binding = os.path.join(OUT_DIR, "torch_binding.o")
    procs.append((BINDING_SOURCE, subprocess.Popen(_binding_command(binding), stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                                                   text=True)))
    failed = []
    for src, pr in procs:
        out, _ = pr.communicate()
        if out and (verbose_ptxas or pr.returncode):
            sys.stderr.write(out)
        if pr.returncode:
            failed.append(src)
    if failed:
        raise RuntimeError(f"compilation failed for {failed}")
    tmp = LIB_PATH + f".tmp{os.getpid()}"
    subprocess.check_call([nvcc(), *ARCH, "-shared", "-o", tmp, *objs])
    os.replace(tmp, LIB_PATH)
    _link_binding(binding)
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose_ptxas="-v" in sys.argv))
