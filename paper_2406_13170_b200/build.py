"""Builds libamph.so (the C-ABI library) in-tree with nvcc for sm_100a, and torch_ops.so (torch tensors to its operators) beside it.

The library needs nvcc alone: `python paper_2406_13170_b200/build.py --library` (or build(ops=False)) leaves out torch_ops.so, which needs
torch's and Python's headers."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SOURCES = ["amph_api.cu", "kernels.cu", "gemm_tc.cu", "gemm_wide.cu", "gemm_rows.cu", "attention_mma.cu", "attention_tc.cu", "project_static.cu",
           "adapters.cu", "paged.cu"]
LIB = os.path.join(HERE, "libamph.so")
OPS = os.path.join(HERE, "torch_ops.so")


def _stale(target: str) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    deps = [os.path.join(HERE, "csrc", f) for f in os.listdir(os.path.join(HERE, "csrc"))]
    deps.append(os.path.join(ROOT, "include", "amph.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False, ops: bool = True) -> str:
    """Builds what is missing or older than its sources; a fault of torch_ops.so is raised once the library is there."""
    make_lib, make_ops = force or _stale(LIB), ops and (force or _stale(OPS))
    running = fault = None
    if make_ops:
        try:
            running = subprocess.Popen(_ops_command())
        except Exception as e:
            fault = e
    try:
        if make_lib:
            subprocess.run(_library_command(verbose), check=True)
    finally:
        rc = running.wait() if running else 0
    if fault or rc:
        raise RuntimeError(f"torch_ops.so was not built ({fault or f'the compiler returned {rc}'}); libamph.so is there") from fault
    return LIB


def _library_command(verbose: bool) -> list:
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
           "-Xcompiler", "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"),
           "-I", os.path.join(HERE, "csrc")]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    return cmd + [os.path.join(HERE, "csrc", s) for s in SOURCES] + ["-o", LIB, "-lcudart"]


def _ops_command() -> list:
    import torch
    from torch.utils import cpp_extension
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    include = [os.path.join(ROOT, "include"), *cpp_extension.include_paths(), os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", *(f"-I{d}" for d in include),
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", os.path.join(HERE, "csrc", "torch_ops.cpp"), "-o", OPS,
            *(f"-L{d}" for d in cpp_extension.library_paths()), f"-L{os.path.join(cuda, 'lib64')}",
            "-ltorch_python", "-ltorch_cuda", "-ltorch_cpu", "-lc10_cuda", "-lc10", "-lcudart"]


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, ops="--library" not in sys.argv))
