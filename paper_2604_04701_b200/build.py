"""Builds libmuxq.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a, and _calls.so (the binding's hot calls)."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmuxq.so")
CALLS = os.path.join(HERE, "_calls.so")
OBJ_DIR = os.path.join(HERE, "_build")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
    "--fmad=false",            # dequantization is two separately rounded multiplies (Eq. 3)
    "-Xcompiler", "-fPIC", "-Xptxas", "-v",
]


def _sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _deps_mtime():
    paths = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    paths.append(os.path.join(HERE, "..", "include", "muxq.h"))
    paths.append(os.path.abspath(__file__))
    return max(os.path.getmtime(p) for p in paths)


MARK = "_calls.so for "


def built_for() -> str:
    """What _calls.so depends on beside its sources: it reads tensors by the layout of the torch that it was compiled against."""
    import torch
    return f"{sys.implementation.cache_tag} torch {torch.__version__} {torch.version.git_version} abi {int(torch.compiled_with_cxx11_abi())}"


def _calls_suit() -> bool:
    """Whether _calls.so, which says so in a string of its own, was built for this Python and this torch (not by importing it)."""
    with open(CALLS, "rb") as f:
        return (MARK + built_for()).encode() + b"\0" in f.read()


def build_calls() -> None:
    """_calls.so: py_calls.c, and py_tensor.cpp against the headers and libraries of the torch that is installed."""
    import torch
    os.makedirs(OBJ_DIR, exist_ok=True)
    home = os.path.dirname(torch.__file__)
    flags = ["-O2", "-Wall", "-fPIC", "-I" + sysconfig.get_paths()["include"], f'-DCALLS_BUILT_FOR="{MARK}{built_for()}"']
    objs = [os.path.join(OBJ_DIR, f) for f in ("py_calls.o", "py_tensor.o")]
    subprocess.check_call([os.environ.get("CC", "gcc"), *flags, "-c", os.path.join(CSRC, "py_calls.c"), "-o", objs[0]])
    cxx = os.environ.get("CXX", "g++")
    subprocess.check_call([cxx, *flags, "-std=c++17", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
                           *("-isystem" + os.path.join(home, "include", d) for d in ("", "torch/csrc/api/include")),
                           "-c", os.path.join(CSRC, "py_tensor.cpp"), "-o", objs[1]])
    tmp = CALLS + f".tmp{os.getpid()}"
    libs = os.path.join(home, "lib")
    subprocess.check_call([cxx, "-shared", *objs, "-L" + libs, "-Wl,-rpath," + libs, "-ltorch_python", "-ltorch_cpu", "-lc10", "-o", tmp])
    os.replace(tmp, CALLS)


def build(force: bool = False, verbose: bool = False) -> str:
    fresh = lambda f: not force and os.path.exists(f) and os.path.getmtime(f) >= _deps_mtime()
    if not fresh(CALLS) or not _calls_suit():
        build_calls()
    if fresh(LIB):
        return LIB
    os.makedirs(OBJ_DIR, exist_ok=True)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    srcs = _sources()
    objs = [os.path.join(OBJ_DIR, os.path.basename(s)[:-3] + ".o") for s in srcs]

    def compile_one(pair):
        src, obj = pair
        r = subprocess.run([nvcc, *NVCC_FLAGS, "-c", src, "-o", obj], capture_output=True, text=True)
        return src, r

    with ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        for src, r in ex.map(compile_one, zip(srcs, objs)):
            if verbose or r.returncode:
                sys.stderr.write(f"--- {os.path.basename(src)}\n{r.stdout}{r.stderr}\n")
            if r.returncode:
                raise RuntimeError(f"nvcc failed on {src}")
    tmp = LIB + f".tmp{os.getpid()}"
    subprocess.check_call([nvcc, "-shared", "-o", tmp, *objs, "-gencode", "arch=compute_100a,code=sm_100a"])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
