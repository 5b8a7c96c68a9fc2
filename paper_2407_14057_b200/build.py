"""Builds the CUDA library in-tree (nvcc, sm_100a only, one shared object) and the argument marshaller beside it."""
from __future__ import annotations

import hashlib
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "liblazyllm.so")
STAMP = os.path.join(HERE, "_build", "stamp.txt")
CALL_SRC = os.path.join(CSRC, "lazycall.cpp")
CALL_LIB = os.path.join(HERE, "lazycall.so")
CALL_STAMP = os.path.join(HERE, "_build", "lazycall.txt")

# No --use_fast_math: it would turn expf and division into approximations everywhere; the kernels
# call the fast intrinsics explicitly where that is wanted.
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-Xptxas", "-v",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _digest() -> str:
    h = hashlib.sha256()
    files = _sources() + sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cuh"))
    files.append(os.path.join(ROOT, "include", "lazyllm.h"))
    for f in files:
        h.update(f.encode())
        with open(f, "rb") as fh:
            h.update(fh.read())
    h.update(" ".join(NVCC_FLAGS).encode())
    return h.hexdigest()


def build_call(force: bool = False) -> str:
    """Compiles csrc/lazycall.cpp, the Python module that marshals tensors, against the installed torch."""
    import sysconfig

    import torch
    from torch.utils.cpp_extension import include_paths
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-o", CALL_LIB, CALL_SRC,
           "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_paths()["include"],
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    cmd += [f"-I{p}" for p in include_paths()]
    cmd += ["-L" + os.path.join(os.path.dirname(torch.__file__), "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]
    h = hashlib.sha256(" ".join(cmd + [torch.__version__]).encode())
    for f in (CALL_SRC, os.path.join(ROOT, "include", "lazyllm.h")):
        with open(f, "rb") as fh:
            h.update(fh.read())
    if not force and os.path.exists(CALL_LIB) and os.path.exists(CALL_STAMP):
        with open(CALL_STAMP) as f:
            if f.read().strip() == h.hexdigest():
                return CALL_LIB
    os.makedirs(os.path.dirname(CALL_STAMP), exist_ok=True)
    made = f"{CALL_LIB}.{os.getpid()}"
    try:
        subprocess.run([made if c == CALL_LIB else c for c in cmd], check=True)
        os.replace(made, CALL_LIB)
    except (OSError, subprocess.CalledProcessError):
        for f in (made, CALL_LIB):  # no marshaller is better than an old one, which could expect other entry points
            if os.path.exists(f):
                os.remove(f)
        raise
    with open(CALL_STAMP, "w") as f:
        f.write(h.hexdigest())
    return CALL_LIB


def build(force: bool = False, verbose: bool = False) -> str:
    """Compiles every .cu under csrc/ and links liblazyllm.so, then the marshaller; returns the library's path.

    The library needs nvcc alone.  The marshaller needs torch, Python's headers and a C++ compiler as well; where one of them is
    missing this says so, and only the Python wrappers that go through it are then missing."""
    path = build_library(force, verbose)
    try:
        build_call(force)
    except (ImportError, OSError, subprocess.CalledProcessError) as e:
        sys.stderr.write(f"{os.path.basename(CALL_LIB)} was not built ({e}): the Python wrappers of the operators on bounded "
                         "and shared caches will raise\n")
    return path


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compiles every .cu under csrc/ and links liblazyllm.so; returns its path."""
    dig = _digest()
    if not force and os.path.exists(LIB) and os.path.exists(STAMP):
        with open(STAMP) as f:
            if f.read().strip() == dig:
                return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    bdir = os.path.join(HERE, "_build")
    os.makedirs(bdir, exist_ok=True)
    objs, procs = [], []
    for src in _sources():
        obj = os.path.join(bdir, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        cmd = [nvcc] + NVCC_FLAGS + ["-c", src, "-o", obj]
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    log = []
    for src, p in procs:
        out, _ = p.communicate()
        log.append(f"== {os.path.basename(src)}\n{out}")
        if p.returncode != 0:
            sys.stderr.write("\n".join(log))
            raise RuntimeError(f"nvcc failed on {src}")
    with open(os.path.join(bdir, "ptxas.log"), "w") as f:
        f.write("\n".join(log))
    if verbose:
        print("\n".join(log))
    cmd = [nvcc, "-shared", "-o", LIB] + objs + ["-gencode", "arch=compute_100a,code=sm_100a"]
    subprocess.run(cmd, check=True)
    with open(STAMP, "w") as f:
        f.write(dig)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
