"""Build libicv.so (HIP, gfx950 only) in-tree with hipcc.

    python -m paper_1907_02129_amd.build

Every .hip file under csrc/ is compiled to an object (in parallel) and linked into
paper_1907_02129_amd/libicv.so.  hipcc cross-compiles without a GPU present.  The host compiler builds
icv_python.cpp, the argument checks of the operators that take torch tensors, into _icv_python.so beside it; libicv.so needs
neither, and is built without it where torch, Python's headers or that compiler are missing.
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libicv.so")
PYTHON_MODULE = os.path.join(PKG, "_icv_python.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
    # the compiler must not form packed-fp32 instructions by itself on the test machines
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def _compile(src: str, verbose: bool, incremental: bool = False) -> str:
    obj = os.path.join(OBJ, os.path.basename(src).replace(".hip", ".o"))
    if incremental and os.path.exists(obj):
        deps = [src] + glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
        if all(os.path.getmtime(d) <= os.path.getmtime(obj) for d in deps):
            return obj
    cmd = [HIPCC, *FLAGS, "-c", src, "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in r.stdout.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{out}")
    if out.strip() and verbose:
        print(out)
    return obj


def missing_for_python_module() -> str:
    """What is not there of the things that only _icv_python.so needs; "" if all are."""
    torch = importlib.util.find_spec("torch")
    if torch is None or not torch.origin:
        return "torch"
    if not os.path.exists(os.path.join(os.path.dirname(torch.origin), "include", "torch", "csrc", "autograd", "python_variable.h")):
        return "torch's headers"
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        return "Python.h"
    cxx = os.environ.get("CXX", "g++")
    return "" if shutil.which(cxx) else cxx


def build_python_module(verbose: bool = False, incremental: bool = False) -> str:
    import torch                                  # its headers and libraries; the module runs in a process that has torch loaded
    src, at = os.path.join(CSRC, "icv_python.cpp"), os.path.dirname(os.path.abspath(torch.__file__))
    deps = [src, os.path.join(ROOT, "include", "icv.h")]
    if incremental and os.path.exists(PYTHON_MODULE) and all(os.path.getmtime(d) <= os.path.getmtime(PYTHON_MODULE) for d in deps):
        return PYTHON_MODULE
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-Wall",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", os.path.join(ROOT, "include"),
           "-isystem", os.path.join(at, "include"), "-isystem", os.path.join(at, "include", "torch", "csrc", "api", "include"),
           "-I", sysconfig.get_paths()["include"], src, "-o", PYTHON_MODULE, "-L", os.path.join(at, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed on {src}:\n{r.stdout}")
    if r.stdout.strip() and verbose:
        print(r.stdout)
    return PYTHON_MODULE


def build(verbose: bool = False, jobs: int = 8, incremental: bool = False) -> str:
    """Compile every source (or, with `incremental`, those newer than their object) and link the library."""
    os.makedirs(OBJ, exist_ok=True)
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.hip")))
    missing = missing_for_python_module()
    with cf.ThreadPoolExecutor(max_workers=min(jobs, len(srcs) + 1)) as ex:
        module = None if missing else ex.submit(build_python_module, verbose, incremental)
        objs = list(ex.map(lambda s: _compile(s, verbose, incremental), srcs))
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    if module:
        module.result()
    else:
        # an old one would check against another description of the structs
        if os.path.exists(PYTHON_MODULE):
            os.remove(PYTHON_MODULE)
        print(f"without _icv_python.so, which needs {missing}: the library's C interface is complete, the operators on sequences and in "
              "8-bit floating point cannot be called through binding.py", file=sys.stderr)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-q" not in sys.argv, incremental="-i" in sys.argv))
