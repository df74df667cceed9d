"""Builds the CUDA library in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import glob
import os
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB_PATH = os.path.join(_HERE, "libattn_fwd.so")
# The same sources with the test hooks compiled in (bounded waits of 1 ms instead of 1 s, and an extra
# entry that makes the producer leave out one K/V load): used by one GPU test to make a wait run out
# and check the time-out status.  Never loaded by the package.
WAIT_TEST_LIB_PATH = os.path.join(_HERE, "libattn_fwd_waittest.so")
# Python extension (see csrc/binding.cpp) that build() makes beside the library.  Where it is missing, as beside a library that was
# built by hand, api.py marshals every call itself.
BINDING_PATH = os.path.join(_HERE, "_binding.so")
WAIT_TEST_FLAGS = ["-DATTN_TEST_HOOKS", "-DATTN_TEST_WAIT_LIMIT_NS=1000000ull"]

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-shared", "-Xcompiler", "-fPIC",
]


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh"))
                  + glob.glob(os.path.join(_HERE, "..", "include", "*.h")))


def is_stale(path: str = LIB_PATH) -> bool:
    if not os.path.exists(path):
        return True
    t = os.path.getmtime(path)
    return any(os.path.getmtime(s) > t for s in _sources())


def _compile(path: str, extra, verbose: bool) -> str:
    nvcc = os.environ.get("NVCC", "nvcc")
    tmp = path + ".tmp.%d" % os.getpid()
    cmd = [nvcc] + NVCC_FLAGS + list(extra) + (["-Xptxas", "-v"] if verbose else []) + [
        "-o", tmp, os.path.join(CSRC, "attn_api.cu")]
    subprocess.check_call(cmd)
    os.replace(tmp, path)
    return path


def build_binding(force: bool = False) -> str:
    """Compile csrc/binding.cpp, the C++ argument marshalling of the latency-bound entry points, against the installed torch."""
    src = os.path.join(CSRC, "binding.cpp")
    header = os.path.join(_HERE, "..", "include", "attn_fwd.h")
    if not force and os.path.exists(BINDING_PATH) and os.path.getmtime(BINDING_PATH) >= max(os.path.getmtime(src), os.path.getmtime(header)):
        return BINDING_PATH
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    torch_lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    cuda = os.environ.get("CUDA_HOME") or cpp_extension.CUDA_HOME or "/usr/local/cuda"
    tmp = BINDING_PATH + ".tmp.%d" % os.getpid()
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden",
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI), "-I", sysconfig.get_paths()["include"]]
    for inc in cpp_extension.include_paths() + [os.path.join(cuda, "include")]:
        cmd += ["-isystem", inc]
    cmd += ["-o", tmp, src, "-L", torch_lib, "-Wl,-rpath," + torch_lib, "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
    subprocess.check_call(cmd)
    os.replace(tmp, BINDING_PATH)
    return BINDING_PATH


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile csrc/attn_api.cu (which includes every kernel header) into libattn_fwd.so, and the Python extension."""
    build_binding(force)
    if not force and not is_stale():
        return LIB_PATH
    return _compile(LIB_PATH, [], verbose)


def build_wait_test(force: bool = False) -> str:
    """Compile the test-hook variant of the library (see WAIT_TEST_LIB_PATH)."""
    if not force and not is_stale(WAIT_TEST_LIB_PATH):
        return WAIT_TEST_LIB_PATH
    return _compile(WAIT_TEST_LIB_PATH, WAIT_TEST_FLAGS, False)


if __name__ == "__main__":
    print(build(force=True, verbose=True))
