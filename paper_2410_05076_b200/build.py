"""Build libtidal.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a, and _fast_call (tensors in, C calls out; see
csrc/fast_call.cpp) with g++ against the installed torch. The library needs neither torch's nor Python's headers and
is built and loaded without the other."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libtidal.so")
SOURCES = ["tidal_api.cu"]
DEPS = ["tidal_api.cu", "attn_kernels.cuh", "block_kernels.cuh", "block_select_kernels.cuh", "block_attn_kernels.cuh", "chunk_kernels.cuh", "evict_kernels.cuh", "page_kernels.cuh", "rope_kernels.cuh", "split_select_kernels.cuh", "topk_kernels.cuh", "weight_kernels.cuh", os.path.join("..", "..", "include", "tidal.h")]


FAST_DEPS = ["fast_call.cpp", os.path.join("..", "..", "include", "tidal.h")]


def fast_path() -> str:
    """The file's name says for which Python and which torch it was built: another one's is not taken for it."""
    import torch
    return os.path.join(HERE, f"_fast_call-torch{torch.__version__}{sysconfig.get_config_var('EXT_SUFFIX')}")


def nvcc_path() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _older(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(os.path.join(CSRC, d)) > t for d in deps)


def is_stale() -> bool:
    return _older(LIB, DEPS)


def fast_is_stale() -> bool:
    return _older(fast_path(), FAST_DEPS)


def build_fast() -> str:
    import torch
    root = os.path.dirname(torch.__file__)
    cuda = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")
    path = fast_path()
    tmp = path + f".tmp{os.getpid()}"
    subprocess.check_call(
        ["g++", "-O2", "-std=c++20", "-shared", "-fPIC", "-fvisibility=hidden", f"-I{os.path.join(root, 'include')}",
         f"-I{sysconfig.get_paths()['include']}", f"-I{cuda}", "-o", tmp, os.path.join(CSRC, "fast_call.cpp"),
         f"-L{os.path.join(root, 'lib')}", "-ltorch_python", "-ltorch_cpu", "-lc10_cuda", "-lc10"])
    os.replace(tmp, path)
    return path


def build(force: bool = False, verbose: bool = False) -> str:
    """libtidal.so, where it is missing or older than its sources."""
    if not force and not is_stale():
        return LIB
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [nvcc_path(), "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
           "-shared", "-Xcompiler", "-fPIC", "-cudart", "static",
           "-o", tmp] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
    print(build_fast() if "--force" in sys.argv or fast_is_stale() else fast_path())
