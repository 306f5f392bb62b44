"""Build libilwdetr.so (the C-ABI of include/ilwdetr.h) for sm_103a with nvcc, in-tree.

Each translation unit is compiled in parallel; the shared library is written next to this file, and beside it
_mxbind.so, the Python binding of the operators in mx.py (host code against torch's headers; where there is no torch,
whose tensors it takes, it is left out).
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libilwdetr.so")
BIND_SRC, BIND = os.path.join(CSRC, "mx_bind.cpp"), os.path.join(HERE, "_mxbind.so")
BIND_KEY = os.path.join(OBJ, "_mxbind.key")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-Xcompiler", "-Wall",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC, "--expt-relaxed-constexpr"]


def nvcc() -> str:
    p = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(p):
        raise RuntimeError("nvcc not found: the CUDA library cannot be built")
    return p


def sources() -> list[str]:
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _stale(out: str, deps: list[str]) -> bool:
    if not os.path.exists(out):
        return True
    t = os.path.getmtime(out)
    return any(os.path.getmtime(d) > t for d in deps)


def importable(name: str) -> bool:
    try:
        __import__(name)
    except ImportError:
        return False
    return True


def binding_key() -> str:
    """What _mxbind.so fits besides its source: this interpreter and this torch."""
    import sysconfig

    import torch

    return " ".join([sysconfig.get_config_var("SOABI") or sys.version, torch.__version__, torch.__path__[0]])


def _read(path: str) -> str:
    return open(path).read() if os.path.exists(path) else ""


def build_binding(verbose: bool = False) -> str:
    """_mxbind.so: one host translation unit, linked with torch's own libraries."""
    import sysconfig

    import torch

    base = torch.__path__[0]
    cuda = os.path.dirname(os.path.dirname(nvcc()))
    tmp = BIND + ".tmp%d" % os.getpid()
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-Wall", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI]
    for d in (sysconfig.get_paths()["include"], os.path.join(base, "include"), os.path.join(cuda, "include")):
        cmd += ["-isystem", d]
    cmd += ["-I", os.path.join(ROOT, "include"), BIND_SRC, "-o", tmp, "-L", os.path.join(base, "lib"), "-Wl,-rpath," + os.path.join(base, "lib"),
            "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
    if verbose:
        print(" ".join(cmd), file=sys.stderr)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed on {os.path.basename(BIND_SRC)}:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, BIND)
    with open(BIND_KEY, "w") as f:
        f.write(binding_key())
    return r.stderr


def build(force: bool = False, verbose: bool = False, extra: list[str] | None = None) -> str:
    os.makedirs(OBJ, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    headers.append(os.path.join(ROOT, "include", "ilwdetr.h"))
    srcs = sources()
    objs = [os.path.join(OBJ, os.path.basename(s)[:-3] + ".o") for s in srcs]
    todo = [(s, o) for s, o in zip(srcs, objs) if force or _stale(o, [s] + headers)]

    def compile_one(so):
        s, o = so
        cmd = [nvcc()] + ARCH + FLAGS + (extra or []) + ["-c", s, "-o", o]
        if verbose:
            print(" ".join(cmd), file=sys.stderr)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {os.path.basename(s)}:\n{r.stdout}\n{r.stderr}")
        return r.stderr

    bind = importable("torch") and (force or _read(BIND_KEY) != binding_key() or _stale(BIND, [BIND_SRC, os.path.join(ROOT, "include", "ilwdetr.h")]))
    with cf.ThreadPoolExecutor(max_workers=min(9, 1 + len(todo))) as ex:
        binding = ex.submit(build_binding, verbose) if bind else None
        for msg in ex.map(compile_one, todo):
            if verbose and msg:
                print(msg, file=sys.stderr)
    if force or todo or _stale(LIB, objs):
        tmp = LIB + ".tmp%d" % os.getpid()
        cmd = [nvcc()] + ARCH + ["-shared", "-Xcompiler", "-fPIC", "-o", tmp] + objs
        subprocess.run(cmd, check=True)
        os.replace(tmp, LIB)
    if binding:
        binding.result()  # (an error of the binding's build leaves the library built)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
