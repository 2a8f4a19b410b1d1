"""Compile the CUDA library in-tree: paper_2008_11343_b200/libapms.so (sm_100a only)."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
# The translation units and what each includes: apms.cu the context and the kernels of the step, operators.cu the op_* files.
UNITS = {"apms.cu": lambda f: not f.startswith("op"), "operators.cu": lambda f: f.startswith("op") or f == "errors.h"}
HDR = os.path.join(ROOT, "include", "apms.h")
BUILD = os.path.join(HERE, "_build")                     # objects of the units
LIB = os.path.join(HERE, "libapms.so")
EXT = os.path.join(HERE, "_operators.so")                # CPython extension: the operators beside the step on torch tensors
EXT_SRC = os.path.join(CSRC, "torch_operators.cpp")
LIB_CHECKED = os.path.join(HERE, "libapms_checked.so")   # the same source with -DAPMS_BOUNDS_CHECK (debugging aid)
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-fmad=false", "-prec-div=true", "-prec-sqrt=true", "-ftz=false",
    "-Xcompiler", "-fPIC", "-Xptxas", "-v",
    "-I", os.path.join(ROOT, "include"),
]


def _sources(unit: str) -> list:
    return [HDR] + [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh", ".h")) and UNITS[unit](f)]


def _older(out: str, sources: list) -> bool:
    return not os.path.exists(out) or os.path.getmtime(out) < max(os.path.getmtime(f) for f in sources)


def is_stale(lib: str = LIB) -> bool:
    return _older(EXT, [HDR, EXT_SRC]) or any(_older(lib, _sources(unit)) for unit in UNITS)


def _extension_command(out: str) -> list:
    import sysconfig

    import torch
    from torch.utils import cpp_extension

    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    include = [os.path.join(ROOT, "include"), sysconfig.get_path("include"), os.path.join(cuda, "include"), *cpp_extension.include_paths()]
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            *(f"-isystem{d}" for d in include), EXT_SRC, "-o", out, *(f"-L{d}" for d in cpp_extension.library_paths()),
            "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch_python"]


def build(force: bool = False, verbose: bool = False, checked: bool = False) -> str:
    """Compile libapms.so, or with checked=True libapms_checked.so (every access of the step's kernels validated on the
    device).  The units are compiled side by side; without `force` only those whose sources are newer than their object."""
    lib = LIB_CHECKED if checked else LIB
    if not force and not is_stale(lib):
        return lib
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    extra = ["-DAPMS_BOUNDS_CHECK"] if checked else []
    pid, running, objects = os.getpid(), [], []
    if not checked and (force or _older(EXT, [HDR, EXT_SRC])):
        running.append((EXT, subprocess.Popen(_extension_command(f"{EXT}.{pid}"), stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for unit in UNITS:
        obj = os.path.join(BUILD, unit.replace(".cu", "_checked.o" if checked else ".o"))
        objects.append(obj)
        if force or _older(obj, _sources(unit)):
            os.makedirs(BUILD, exist_ok=True)
            cmd = [nvcc, *NVCC_FLAGS, *extra, "-c", os.path.join(CSRC, unit), "-o", f"{obj}.{pid}"]
            running.append((obj, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for obj, proc in running:
        said = proc.communicate()[0]
        if verbose or proc.returncode != 0:
            sys.stderr.write(said)
        if proc.returncode != 0:
            raise RuntimeError(f"nvcc failed building {os.path.basename(obj)}")
        os.replace(f"{obj}.{pid}", obj)
    tmp = lib + f".tmp{pid}"
    proc = subprocess.run([nvcc, *NVCC_FLAGS[:2], "-shared", *objects, "-o", tmp], capture_output=True, text=True)
    if proc.returncode != 0:
        sys.stderr.write(proc.stdout + proc.stderr)
        raise RuntimeError(f"nvcc failed linking {os.path.basename(lib)}")
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    print(build(force=True, verbose=True))
    if "--checked" in sys.argv:
        print(build(force=True, checked=True))
