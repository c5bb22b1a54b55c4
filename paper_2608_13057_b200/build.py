"""Builds libtempo.so (the C-ABI CUDA library, nvcc for sm_100a) and _marshal (the Python module that marshals the short
calls, the host compiler against torch's headers) in-tree."""
from __future__ import annotations

import importlib.metadata
import importlib.util
import os
import subprocess
import sys
import sysconfig

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libtempo.so")
SOURCES = ["api.cu", "dispatch.cu", "dispatch_sampled.cu", "permute.cu", "ffn.cu", "combine.cu", "pack.cu",
           "norm.cu", "route.cu", "few.cu"]


MARSHAL_SRC = os.path.join(CSRC, "marshal.cpp")
MARSHAL_PATH = os.path.join(PKG_DIR, "_marshal" + sysconfig.get_config_var("EXT_SUFFIX"))
HEADER = os.path.join(ROOT, "include", "tempo.h")


def _stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if not f.endswith(".cpp")] + [HEADER]
    return any(os.path.getmtime(d) > t for d in deps)


def _torch_dir() -> str:
    return os.path.dirname(os.path.abspath(importlib.util.find_spec("torch").origin))


def _marshal_stale(built_for: str) -> bool:
    """Whether the module is missing, older than its sources or built against another torch, which its own text tells."""
    if not os.path.exists(MARSHAL_PATH) or \
            os.path.getmtime(MARSHAL_PATH) < max(os.path.getmtime(MARSHAL_SRC), os.path.getmtime(HEADER)):
        return True
    with open(MARSHAL_PATH, "rb") as f:
        return f"(built for {built_for})".encode() not in f.read()


def build_marshal(force: bool = False) -> str:
    """The extension links torch's libraries by name only: importing torch first loads them."""
    base = _torch_dir()
    built_for = f"torch {importlib.metadata.version('torch')} in {base}"
    if not force and not _marshal_stale(built_for):
        return MARSHAL_PATH
    import torch
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DTEMPO_BUILT_FOR="{built_for}"',
           "-I", os.path.join(ROOT, "include"), "-isystem", os.path.join(base, "include"),
           "-isystem", os.path.join(base, "include", "torch", "csrc", "api", "include"),
           "-isystem", os.path.join(cuda, "include"), "-isystem", sysconfig.get_paths()["include"],
           "-o", MARSHAL_PATH, MARSHAL_SRC, "-L", os.path.join(base, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("the host compiler failed building _marshal")
    return MARSHAL_PATH


def build(force: bool = False, verbose: bool = False) -> str:
    build_marshal(force)
    if not force and not _stale():
        return LIB_PATH
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
           "-Xcompiler", "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-o", LIB_PATH] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("nvcc failed building libtempo.so")
    if verbose:
        print(res.stdout + res.stderr)
    return LIB_PATH


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
