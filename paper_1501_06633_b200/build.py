"""In-tree build of ``libmaxdnn.so`` (nvcc, sm_100a only).

``python -m paper_1501_06633_b200.build`` compiles the CUDA sources under
``csrc/`` into ``paper_1501_06633_b200/libmaxdnn.so``.  nvcc cross-compiles, so
no GPU is needed to build.
"""
from __future__ import annotations

import glob
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmaxdnn.so")
SOURCES = ["maxdnn_api.cu", "train8_api.cu", "norm_api.cu", "gemm8_api.cu", "plan.cpp", "gemm8_plan.cpp"]
NVCC_FLAGS = ["-std=c++17", "-O3", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC", "-shared", "-cudart", "static", "--threads", "0"]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = glob.glob(os.path.join(CSRC, "*")) + [os.path.join(HERE, "..", "include", "maxdnn.h"),
                                                 os.path.abspath(__file__)]
    return any(os.path.getmtime(p) > t for p in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile if the library is missing or older than its sources; return its path."""
    if force or _stale():
        nvcc = os.environ.get("NVCC", "nvcc")
        tmp = LIB + ".tmp.%d" % os.getpid()
        extra = os.environ.get("MAXDNN_NVCC_EXTRA", "").split()
        cmd = [nvcc] + NVCC_FLAGS + extra + (["-Xptxas", "-v"] if verbose else []) + ["-o", tmp] + \
              [os.path.join(CSRC, s) for s in SOURCES]
        res = subprocess.run(cmd, capture_output=True, text=True)
        if verbose:
            sys.stderr.write(res.stdout + res.stderr)
        if res.returncode != 0:
            if os.path.exists(tmp):
                os.remove(tmp)
            raise RuntimeError("nvcc failed:\n%s\n%s" % (" ".join(cmd), res.stdout + res.stderr))
        os.replace(tmp, LIB)
    return LIB


BINDING = os.path.join(HERE, "_train8.so")
BINDING_SOURCE = os.path.join(CSRC, "train8_binding.cpp")


def build_binding(force: bool = False) -> str:
    """Compile the marshalling module of the 8-bit training operators (host C++ against the
    installed torch's headers) if it is missing or older than its sources; return its path."""
    deps = (BINDING_SOURCE, os.path.join(HERE, "..", "include", "maxdnn.h"), os.path.abspath(__file__))
    if not force and os.path.exists(BINDING) and all(os.path.getmtime(p) <= os.path.getmtime(BINDING) for p in deps):
        return BINDING
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    tmp = BINDING + ".tmp.%d" % os.getpid()
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    cmd = [os.environ.get("CXX", "g++"), "-std=c++17", "-O2", "-fPIC", "-shared", "-w",
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI), "-I" + sysconfig.get_paths()["include"],
           "-I" + os.path.join(cuda, "include")] + ["-I" + p for p in cpp_extension.include_paths()] + \
          ["-o", tmp, BINDING_SOURCE, "-L" + libs, "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        if os.path.exists(tmp):
            os.remove(tmp)
        raise RuntimeError("compiling the binding failed:\n%s\n%s" % (" ".join(cmd), res.stdout + res.stderr))
    os.replace(tmp, BINDING)
    return BINDING


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
    print(build_binding(force="--force" in sys.argv))
