"""Build the CUDA library (sm_100a) in-tree with nvcc.

`python -m paper_2602_08329_b200.build` compiles csrc/prhs.cu into libprhs.so next to
this file (nvcc cross-compiles without a GPU) and csrc/marshal.cpp, the compiled part of the
binding, into _marshal.so.
"""
from __future__ import annotations

import importlib.metadata
import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libprhs.so")
MARSHAL = os.path.join(HERE, "_marshal.so")
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
         "-Xcompiler", "-fPIC", "-shared"]


def sources():
    out = [os.path.join(CSRC, f) for f in sorted(os.listdir(CSRC)) if f != "marshal.cpp"]
    return out + [os.path.join(os.path.dirname(HERE), "include", "prhs.h")]


def _older(target: str, inputs) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(s) > t for s in inputs)


def stale() -> bool:
    return _older(LIB, sources()) or _marshal_stale()


def marshal_sources():
    return [os.path.join(CSRC, "marshal.cpp"), os.path.join(os.path.dirname(HERE), "include", "prhs.h")]


def _built_for():
    """What _marshal.so has to fit, as the text that it carries; None without torch (and so without a use for it)."""
    if importlib.util.find_spec("torch") is None:
        return None
    try:
        version = importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:       # a source tree on the path
        import torch
        version = torch.__version__
    return f"for torch {version}, python {sys.version_info.major}.{sys.version_info.minor};"


def _marshal_stale() -> bool:
    wanted = _built_for()
    if wanted is None:
        return False
    if _older(MARSHAL, marshal_sources()):
        return True
    with open(MARSHAL, "rb") as f:
        return wanted.encode() not in f.read()


def _run(cmd, what: str) -> str:
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"{what} failed:\n" + res.stdout + res.stderr)
    return res.stderr


def build_marshal(force: bool = False) -> str:
    """The extension links the torch libraries that the process has loaded anyway (no search path is recorded).

    It is built again for another torch or python.  Where there is no torch there is no Python binding either, and the C
    library is built alone.
    """
    src = os.path.join(CSRC, "marshal.cpp")
    wanted = _built_for()
    if wanted is not None and (force or _marshal_stale()):
        import torch
        root = os.path.dirname(torch.__file__)
        inc = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
               sysconfig.get_paths()["include"]]
        _run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared",
              f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DPRHS_BUILT_FOR="{wanted}"'] + [f"-I{p}" for p in inc] +
             ["-o", MARSHAL, src, "-L" + os.path.join(root, "lib"), "-lc10", "-ltorch_cpu", "-ltorch", "-ltorch_python"], "g++")
    return MARSHAL


def build(force: bool = False, verbose: bool = False, nvtx: bool = False) -> str:
    """nvtx=True (`--nvtx`) puts every launch in an NVTX range named after its stage."""
    build_marshal(force)
    if not force and not _older(LIB, sources()):
        return LIB
    log = _run([NVCC] + FLAGS + (["-Xptxas", "-v"] if verbose else []) + (["-DPRHS_NVTX", "-ldl"] if nvtx else []) +
               ["-o", LIB, os.path.join(CSRC, "prhs.cu")], "nvcc")
    if verbose:
        print(log)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv, nvtx="--nvtx" in sys.argv))
