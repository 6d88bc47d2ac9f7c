"""Compile libflexdraft.so (all CUDA kernels + the C ABI) for sm_100a with nvcc, and the binding's native argument
marshalling with gcc (where there are gcc and Python's headers), in-tree."""
from __future__ import annotations

import glob
import os
import subprocess
import sysconfig
import warnings

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SO = os.path.join(HERE, "libflexdraft.so")
MARSHAL_SRC = os.path.join(HERE, "csrc", "marshal.c")
MARSHAL = os.path.join(HERE, "_marshal" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
NVCC_FLAGS = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC", "-shared"]


def sources():
    return sorted(glob.glob(os.path.join(HERE, "csrc", "*.cu")))


def _stale() -> bool:
    if not os.path.exists(SO):
        return True
    t = os.path.getmtime(SO)
    deps = sources() + glob.glob(os.path.join(HERE, "csrc", "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    return any(os.path.getmtime(f) > t for f in deps)


def build_marshal(force: bool = False) -> str:
    """The native argument marshalling of the binding (a CPython extension, no CUDA).  Returns its path."""
    if force or not os.path.exists(MARSHAL) or os.path.getmtime(MARSHAL) < os.path.getmtime(MARSHAL_SRC):
        tmp = MARSHAL + f".tmp{os.getpid()}"
        subprocess.run(["gcc", "-O2", "-shared", "-fPIC", "-I", sysconfig.get_paths()["include"], "-o", tmp, MARSHAL_SRC, "-ldl"], check=True)
        os.replace(tmp, MARSHAL)
    return MARSHAL


def build(force: bool = False, verbose: bool = False) -> str:
    """Build if the library is missing or older than a source.  Returns its path."""
    if force or _stale():
        nvcc = os.environ.get("NVCC", "nvcc")
        tmp = SO + f".tmp{os.getpid()}"
        cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + \
              ["-I", os.path.join(ROOT, "include"), "-o", tmp] + sources()
        subprocess.run(cmd, check=True)
        os.replace(tmp, SO)
    try:
        build_marshal(force)
    except (OSError, subprocess.CalledProcessError) as e:
        warnings.warn(f"no native argument marshalling ({e}): the binding marshals through ctypes")
    return SO


if __name__ == "__main__":
    print(build(force=True, verbose=True))
