"""Builds, in-tree, the C-ABI shared library (CUDA kernels + host planner) for sm_100a with nvcc, and the operators'
argument marshalling with g++."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB_DIR = os.path.join(PKG, "lib")
LIB_PATH = os.path.join(LIB_DIR, "libcleave.so")
SOURCES = ["planner.cpp", "kernels.cu", "kernels_pair.cu", "kernels_verify.cu", "kernels_simple.cu", "api.cu",
           "kernels_adamw.cu", "kernels_norm.cu", "kernels_act.cu", "kernels_linear.cu", "ops.cu"]
HEADERS = ["plan_internal.hpp", "kernels.cuh", "ptx.cuh", "ops.cuh", os.path.join(ROOT, "include", "cleave.h")]


MARSHAL_SOURCE = os.path.join(CSRC, "marshal.cpp")
MARSHAL_PATH = os.path.join(PKG, "_marshal" + sysconfig.get_config_var("EXT_SUFFIX"))


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def is_stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + [h if os.path.isabs(h) else os.path.join(CSRC, h) for h in HEADERS]
    return any(os.path.getmtime(d) > t for d in deps)


def _marshal_torch() -> str:
    """Path of the note of the torch version that the marshalling was built against (it binds torch's ABI)."""
    return MARSHAL_PATH + ".torch"


def _marshal_is_stale() -> bool:
    import torch
    try:
        with open(_marshal_torch()) as f:
            if f.read() != torch.__version__:
                return True
    except OSError:
        return True
    deps = [MARSHAL_SOURCE, os.path.join(ROOT, "include", "cleave.h")]
    return not os.path.exists(MARSHAL_PATH) or any(os.path.getmtime(d) > os.path.getmtime(MARSHAL_PATH) for d in deps)


def _build_marshal() -> None:
    """Compiles csrc/marshal.cpp, the operators' argument marshalling, against torch's headers (once libcleave.so exists)."""
    import torch
    base = os.path.dirname(torch.__file__)
    cuda = os.path.join(os.path.dirname(os.path.dirname(_nvcc())) or "/usr/local/cuda", "include")
    cmd = ["g++", "-std=c++17", "-O2", "-fPIC", "-shared", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    for d in (os.path.join(base, "include"), os.path.join(base, "include", "torch", "csrc", "api", "include"), cuda, sysconfig.get_paths()["include"]):
        cmd += ["-isystem", d]
    cmd += ["-I", os.path.join(ROOT, "include"), MARSHAL_SOURCE, "-o", MARSHAL_PATH, "-L", LIB_DIR, "-l:libcleave.so", "-Wl,-rpath,$ORIGIN/lib",
            "-L", os.path.join(base, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("g++ failed:\n" + res.stdout + res.stderr)
    with open(_marshal_torch(), "w") as f:
        f.write(torch.__version__)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compiles csrc/ into lib/libcleave.so and the binding's marshalling (each only when a source is newer)."""
    if force or is_stale():
        _build_cuda(verbose)
    if force or _marshal_is_stale():
        _build_marshal()
    return LIB_PATH


def _build_cuda(verbose: bool) -> None:
    os.makedirs(LIB_DIR, exist_ok=True)
    cmd = [_nvcc(), "-std=c++17", "-O3", "-lineinfo", "-gencode", "arch=compute_100a,code=sm_100a",
           "--threads", "0", "-shared", "-Xcompiler", "-fPIC,-fvisibility=hidden", "-cudart", "static",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", LIB_PATH]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    if verbose:
        print(res.stderr)


if __name__ == "__main__":
    print(build_library(force=True, verbose="-v" in sys.argv))
