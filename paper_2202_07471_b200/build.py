"""Compile the CUDA library for sm_100a into paper_2202_07471_b200/libsquant.so (in-tree)."""
from __future__ import annotations

import glob
import os
import shutil
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsquant.so")
LIB_DEBUG = os.path.join(HERE, "libsquant_debug.so")   # the checked build (-DSQUANT_DEBUG_BOUNDS), for tests on small cases
OBJECTS = os.path.join(HERE, "_build")
SHARED = [os.path.join(ROOT, "include", "squant.h"), os.path.join(CSRC, "squant_host.h")]
# each translation unit with its headers: the quantizer, the linear operators, the key/value cache
UNITS = [(os.path.join(CSRC, unit + ".cu"), sorted(glob.glob(os.path.join(CSRC, unit + "_*.cuh")))) for unit in ("squant", "linear", "cache")]
UNITS[2][1].append(os.path.join(CSRC, "linear_device.cuh"))
DEPS = [d for source, headers in UNITS for d in (source, *headers)] + SHARED

# -fmad=false: the solver's fp32 steps (division, rounding, difference) are written with
# explicit round-to-nearest intrinsics; no contraction is wanted anywhere else either.
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
              "-fmad=false", "-Xcompiler", "-fPIC", "-Xptxas", "-v",
              "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def nvcc_path() -> str:
    p = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(p):
        raise RuntimeError("nvcc not found: the CUDA library cannot be built")
    return p


def _newer(built: str, sources) -> bool:
    return os.path.exists(built) and all(os.path.getmtime(built) >= os.path.getmtime(d) for d in sources)


def build(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    lib = LIB_DEBUG if debug else LIB
    if not force and _newer(lib, DEPS):
        return lib
    os.makedirs(OBJECTS, exist_ok=True)
    running, objects = [], []
    for source, headers in UNITS:   # side by side: each takes most of a minute
        name = os.path.splitext(os.path.basename(source))[0] + ("_debug" if debug else "")
        obj = os.path.join(OBJECTS, name + ".o")
        objects.append(obj)
        if not force and _newer(obj, [source, *headers, *SHARED]):
            continue
        tmp = obj + f".tmp{os.getpid()}.o"
        cmd = [nvcc_path(), *NVCC_FLAGS, *(["-DSQUANT_DEBUG_BOUNDS"] if debug else []), "-c", "-o", tmp, source]
        running.append((subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True), tmp, obj))
    failed = False
    for process, tmp, obj in running:
        text, _ = process.communicate()
        if verbose or process.returncode != 0:
            print(text)
        if process.returncode != 0:
            failed = True
        else:
            os.replace(tmp, obj)
    if failed:
        raise RuntimeError("nvcc failed building " + os.path.basename(lib))
    tmp = lib + f".tmp{os.getpid()}"
    res = subprocess.run([nvcc_path(), "-gencode", "arch=compute_100a,code=sm_100a", "--shared", "-Xcompiler", "-fPIC", "-o", tmp, *objects],
                         capture_output=True, text=True)
    if res.returncode != 0:
        print(res.stdout)
        print(res.stderr)
        raise RuntimeError("nvcc failed linking " + os.path.basename(lib))
    os.replace(tmp, lib)
    return lib


MARSHAL = os.path.join(HERE, "_marshal.so")            # Python extension: descriptors of LayerBuffers objects
MARSHAL_SRC = os.path.join(CSRC, "marshal.cpp")


def build_marshal(force: bool = False) -> str:
    if not force and os.path.exists(MARSHAL) and all(
            os.path.getmtime(MARSHAL) >= os.path.getmtime(d) for d in (MARSHAL_SRC, os.path.join(ROOT, "include", "squant.h"))):
        return MARSHAL
    import sysconfig
    import torch
    base = os.path.dirname(torch.__file__)
    tmp = MARSHAL + f".tmp{os.getpid()}"
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_paths()["include"],
           "-isystem", os.path.join(base, "include"), "-isystem", os.path.join(base, "include", "torch", "csrc", "api", "include"),
           "-o", tmp, MARSHAL_SRC, "-L", os.path.join(base, "lib"), "-lc10", "-ltorch_cpu", "-ltorch_python"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        print(res.stdout)
        print(res.stderr)
        raise RuntimeError("g++ failed building _marshal.so")
    os.replace(tmp, MARSHAL)
    return MARSHAL


if __name__ == "__main__":
    print(build(force=True, verbose=True))
    print(build_marshal(force=True))
    print(build(force=True, debug=True))
