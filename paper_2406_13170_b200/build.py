"""Builds libamph.so (the C-ABI library) in-tree with nvcc for sm_100a, and torch_ops.so (torch tensors to its operators) beside it."""
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


def _stale() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(OPS):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(OPS))
    deps = [os.path.join(HERE, "csrc", f) for f in os.listdir(os.path.join(HERE, "csrc"))]
    deps.append(os.path.join(ROOT, "include", "amph.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
           "-Xcompiler", "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"),
           "-I", os.path.join(HERE, "csrc")]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(HERE, "csrc", s) for s in SOURCES] + ["-o", LIB, "-lcudart"]
    ops = subprocess.Popen(_ops_command())
    try:
        subprocess.run(cmd, check=True)
    finally:
        rc = ops.wait()
    if rc:
        raise subprocess.CalledProcessError(rc, ops.args)
    return LIB


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
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
