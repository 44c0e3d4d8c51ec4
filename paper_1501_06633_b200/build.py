"""In-tree build of ``libmaxdnn.so`` (nvcc, sm_100a only).

``python -m paper_1501_06633_b200.build`` compiles the CUDA sources under
``csrc/`` into ``paper_1501_06633_b200/libmaxdnn.so``.  nvcc cross-compiles, so
no GPU is needed to build.
"""
from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sys
import warnings

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmaxdnn.so")
SOURCES = ["maxdnn_api.cu", "train8_api.cu", "norm_api.cu", "rms_api.cu", "logprob_api.cu", "gemm8_api.cu", "ortho_api.cu",
           "plan.cpp", "gemm8_plan.cpp", "ortho_plan.cpp"]
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


def _binding_marker(torch_version: str) -> bytes:
    return b"built for torch " + torch_version.encode()


def binding_stale(torch_version: str) -> bool:
    """Whether the marshalling module is missing, older than its sources, or built against another
    torch (it reads tensors through torch's headers)."""
    deps = (BINDING_SOURCE, os.path.join(HERE, "..", "include", "maxdnn.h"), os.path.abspath(__file__))
    if not os.path.exists(BINDING) or any(os.path.getmtime(p) > os.path.getmtime(BINDING) for p in deps):
        return True
    with open(BINDING, "rb") as f:
        return _binding_marker(torch_version) + b"\0" not in f.read()


def build_binding(force: bool = False):
    """Compile the marshalling module of the 8-bit training operators (host C++ against the
    installed torch's headers) if it is stale; return its path.  The operators work without it (their calls
    then take a few microseconds more): None, with a warning, where a compiler or headers are missing."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    if not force and not binding_stale(torch.__version__):
        return BINDING
    cxx, python_include = os.environ.get("CXX", "g++"), sysconfig.get_paths()["include"]
    includes = cpp_extension.include_paths()
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    missing = [] if shutil.which(cxx) else [cxx]
    for header, dirs in (("Python.h", [python_include]), ("torch/csrc/autograd/python_variable.h", includes),
                         ("cuda_runtime_api.h", [os.path.join(cuda, "include")])):
        if not any(os.path.exists(os.path.join(d, header)) for d in dirs):
            missing.append(header)
    if missing:
        warnings.warn("the marshalling module of the 8-bit operators is not built: no " + ", ".join(missing))
        return None
    tmp = BINDING + ".tmp.%d" % os.getpid()
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    cmd = [cxx, "-std=c++17", "-O2", "-fPIC", "-shared", "-w",
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI), "-I" + python_include,
           "-DMAXDNN_BUILT_FOR=\"%s\"" % _binding_marker(torch.__version__).decode(),
           "-I" + os.path.join(cuda, "include")] + ["-I" + p for p in includes] + \
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
    print(build_binding(force="--force" in sys.argv) or "(no marshalling module)")
