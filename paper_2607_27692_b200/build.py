"""Compile in-tree: the CUDA library ``csrc/*.cu`` -> ``libretopk.so`` (sm_100a) and, where torch for CUDA is installed,
its torch binding ``csrc/paged_binding.cpp`` -> ``_paged.so``."""
from __future__ import annotations

import fcntl
import os
import shutil
import subprocess
import sys
import sysconfig

_PKG = os.path.dirname(os.path.abspath(__file__))
SRC_DIR = os.path.join(_PKG, "csrc")
LIB_PATH = os.path.join(_PKG, "libretopk.so")
BINDING_SRC = os.path.join(SRC_DIR, "paged_binding.cpp")
BINDING_PATH = os.path.join(_PKG, "_paged.so")
BINDING_STAMP = BINDING_PATH + ".stamp"      # what the binding was compiled against
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
              "-shared", "-Xcompiler", "-fPIC"]


def _sources():
    return sorted(os.path.join(SRC_DIR, f) for f in os.listdir(SRC_DIR)
                  if f.endswith((".cu", ".cuh"))) + [os.path.join(os.path.dirname(_PKG), "include", "retopk.h")]


def _older(path: str, sources) -> bool:
    if not os.path.exists(path):
        return True
    built = os.path.getmtime(path)
    return any(os.path.getmtime(s) > built for s in sources)


def is_stale() -> bool:
    return _older(LIB_PATH, _sources())


def has_torch() -> bool:
    """Whether there is a torch to bind to: one for CUDA."""
    try:
        import torch
    except ImportError:
        return False
    return torch.version.cuda is not None


def binding_target() -> str:
    """Python's and torch's binary interface: a binding of another one does not load, or worse."""
    import torch
    return f"{sys.implementation.cache_tag} torch {torch.__version__} cxx11 {int(torch._C._GLIBCXX_USE_CXX11_ABI)}"


def _stamp() -> str:
    if not os.path.exists(BINDING_STAMP):
        return ""
    with open(BINDING_STAMP) as f:
        return f.read().strip()


def binding_is_stale() -> bool:
    """False, too, where there is no torch to bind to."""
    return has_torch() and (_older(BINDING_PATH, [BINDING_SRC, _sources()[-1]]) or _stamp() != binding_target())


def find_nvcc() -> str:
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        raise RuntimeError("nvcc not found: cannot build libretopk.so")
    return nvcc


def _build_binding():
    """Host code against torch's headers; its libraries are those that ``import torch`` has loaded."""
    import torch
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        raise RuntimeError("g++ not found: cannot build _paged.so")
    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(find_nvcc()))
    include = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
               os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    tmp = f"{BINDING_PATH}.{os.getpid()}.tmp"
    cmd = [cxx, "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           f'-DBUILT_FOR="{binding_target()}"']
    cmd += ["-I" + d for d in include] + [BINDING_SRC, "-o", tmp, "-L" + os.path.join(root, "lib"), "-L" + _PKG]
    cmd += ["-l:libretopk.so", "-lc10", "-lc10_cuda", "-ltorch", "-ltorch_cpu", "-ltorch_python", "-Wl,-rpath,$ORIGIN"]
    subprocess.run(cmd, check=True)
    if os.path.exists(BINDING_STAMP):
        os.remove(BINDING_STAMP)
    os.replace(tmp, BINDING_PATH)
    with open(tmp, "w") as f:
        f.write(binding_target() + "\n")
    os.replace(tmp, BINDING_STAMP)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile what is missing or older than its sources; return the library's path.

    Several processes may call this at once (one rank per GPU): the check and the build run
    under a file lock, and the library appears under its final name in one rename.
    """
    if not force and not is_stale() and not binding_is_stale():
        return LIB_PATH
    with open(LIB_PATH + ".lock", "w") as lock:
        fcntl.flock(lock, fcntl.LOCK_EX)
        try:
            if force or is_stale():          # another process may have built it meanwhile
                nvcc = find_nvcc()
                units = [s for s in _sources() if s.endswith(".cu")]
                tmp = f"{LIB_PATH}.{os.getpid()}.tmp"
                cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-o", tmp] + units
                subprocess.run(cmd, check=True)
                os.replace(tmp, LIB_PATH)
            if has_torch() and (force or binding_is_stale()):
                _build_binding()
        finally:
            fcntl.flock(lock, fcntl.LOCK_UN)
    return LIB_PATH


if __name__ == "__main__":
    print(build(force=True, verbose=True))
