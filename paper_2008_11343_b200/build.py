"""Compile the CUDA library in-tree: paper_2008_11343_b200/libapms.so (sm_100a only), and the torch extension _operators.so.

The library needs nvcc alone.  The extension needs g++ and torch's headers too, and fits the torch it was built with: where it cannot be
built the library is there all the same, no older extension is left behind, and operators.py raises ImportError when it is used."""
from __future__ import annotations

import os
import signal
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
# The translation units and what each includes: apms.cu the context and the kernels of the step, operators.cu the op_* files, layers.cu the layer* files.
UNITS = {"apms.cu": lambda f: not f.startswith(("op", "layer")), "operators.cu": lambda f: f.startswith("op") or f == "errors.h",
         "layers.cu": lambda f: f.startswith("layer") or f in ("op_common.cuh", "errors.h")}
HDR = os.path.join(ROOT, "include", "apms.h")
BUILD = os.path.join(HERE, "_build")                     # objects of the units
LIB = os.path.join(HERE, "libapms.so")
EXT = os.path.join(HERE, "_operators.so")                # CPython extension: the operators beside the step on torch tensors
EXT_SRC = os.path.join(CSRC, "torch_operators.cpp")
EXT_FOR = os.path.join(BUILD, "operators_built_for.txt")  # the torch and python that the extension was compiled against
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


def _torch_version() -> str:
    from importlib import metadata

    try:
        return metadata.version("torch")
    except metadata.PackageNotFoundError:
        return ""


def _built_for() -> str:
    return f"torch {_torch_version()}, python {sys.version_info.major}.{sys.version_info.minor}\n"


def _extension_stale() -> bool:
    if _older(EXT, [HDR, EXT_SRC]) or not os.path.exists(EXT_FOR):
        return True
    with open(EXT_FOR) as f:
        return f.read() != _built_for()


def is_stale(lib: str = "") -> bool:
    lib = lib or LIB
    return any(_older(lib, _sources(unit)) for unit in UNITS) or (lib == LIB and _extension_stale())


def _extension_command(out: str) -> list:
    import sysconfig

    import torch
    from torch.utils import cpp_extension

    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    include = [os.path.join(ROOT, "include"), sysconfig.get_path("include"), os.path.join(cuda, "include"), *cpp_extension.include_paths()]
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            *(f"-isystem{d}" for d in include), EXT_SRC, "-o", out, *(f"-L{d}" for d in cpp_extension.library_paths()),
            "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch_python"]


def _start(cmd: list) -> subprocess.Popen:
    return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, start_new_session=True)


def _start_extension(out: str):
    """The running compiler, or why there is none."""
    try:
        return _start(_extension_command(out)), ""
    except (ImportError, OSError) as e:                      # no torch, no g++
        return None, f"{type(e).__name__}: {e}"


def build(force: bool = False, verbose: bool = False, checked: bool = False) -> str:
    """Compile libapms.so and _operators.so, or with checked=True libapms_checked.so (every access of the step's kernels validated on
    the device).  The units are compiled side by side; without `force` only those whose sources are newer than their object."""
    lib = LIB_CHECKED if checked else LIB
    if not force and not is_stale(lib):
        return lib
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    extra = ["-DAPMS_BOUNDS_CHECK"] if checked else []
    os.makedirs(BUILD, exist_ok=True)
    pid, running, objects, made = os.getpid(), [], [], []

    def finish(proc, tool, out):
        said = proc.communicate()[0]
        if verbose or proc.returncode != 0:
            sys.stderr.write(said)
        if proc.returncode != 0:
            raise RuntimeError(f"{tool} failed building {os.path.basename(out)}")
        os.replace(f"{out}.tmp{pid}", out)

    extension, why = None, ""
    try:
        if not checked and (force or _extension_stale()):
            made.append(EXT)
            extension, why = _start_extension(f"{EXT}.tmp{pid}")
            running += [extension] if extension else []
        for unit in UNITS:
            obj = os.path.join(BUILD, unit.replace(".cu", "_checked.o" if checked else ".o"))
            objects.append(obj)
            if force or _older(obj, _sources(unit)):
                made.append(obj)
                running.append(_start([nvcc, *NVCC_FLAGS, *extra, "-c", os.path.join(CSRC, unit), "-o", f"{obj}.tmp{pid}"]))
        units = [obj for obj in made if obj != EXT]
        for obj, proc in zip(units, [p for p in running if p is not extension]):
            finish(proc, "nvcc", obj)
        if force or units or any(_older(lib, [obj]) for obj in objects):
            made.append(lib)
            link = _start([nvcc, *NVCC_FLAGS[:2], "-shared", *objects, "-o", f"{lib}.tmp{pid}"])
            running.append(link)
            finish(link, "nvcc", lib)
        if EXT in made:
            try:
                if extension is None:
                    raise RuntimeError(why)
                finish(extension, "g++", EXT)
                with open(EXT_FOR, "w") as f:
                    f.write(_built_for())
            except RuntimeError as e:
                for old in (EXT, EXT_FOR):                   # one that no longer fits is worse than none
                    if os.path.exists(old):
                        os.remove(old)
                sys.stderr.write(f"_operators.so is not built, so paper_2008_11343_b200.operators cannot be used: {e}\n")
    finally:
        for proc in running:                                 # left over where another one failed
            if proc.poll() is None:
                os.killpg(proc.pid, signal.SIGKILL)          # with the passes that it has started
                proc.communicate()
        for out in made:
            if os.path.exists(f"{out}.tmp{pid}"):
                os.remove(f"{out}.tmp{pid}")
    return lib


if __name__ == "__main__":
    print(build(force=True, verbose=True))
    if "--checked" in sys.argv:
        print(build(force=True, checked=True))
