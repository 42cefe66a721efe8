"""Build the CUDA library in-tree: ``python -m paper_2609_19758_b200.build``.

Compiles every ``csrc/*.cu`` for sm_100a with nvcc into ``libfpsk.so`` next to this file, then ``csrc/binding.cpp`` with g++ into
the Python module ``_binding.so``.  The library alone is the whole C ABI and wants nvcc alone: where torch, its headers, Python's or
g++ are missing, the binding is left out with a note (and ``attention.py`` raises).
"""
from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sys
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libfpsk.so")
LIB_BOUNDS = os.path.join(HERE, "libfpsk_bounds.so")       # the same sources with -DFPSK_DEBUG_BOUNDS (index checks)
BINDING = os.path.join(HERE, "_binding.so")


def nvcc_path() -> str:
    p = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(p):
        raise RuntimeError("nvcc not found")
    return p


def sources():
    return sorted(glob.glob(os.path.join(HERE, "csrc", "*.cu")))


def binding_mark() -> str:
    """What a binding carries in its code: the torch and the Python that it is made against."""
    import torch
    return f"fpsk binding for torch {torch.__version__}, python {sys.version_info[0]}.{sys.version_info[1]};"


def binding_is_current() -> bool:
    with open(BINDING, "rb") as f:
        return binding_mark().encode() in f.read()


def needs_build(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    if lib == BINDING:
        sources_ = [os.path.join(HERE, "csrc", "binding.cpp"), os.path.join(ROOT, "include", "fpsk_attention.h")]
        return any(os.path.getmtime(d) > t for d in sources_) or not binding_is_current()
    deps = sources() + glob.glob(os.path.join(HERE, "csrc", "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def binding_lacks() -> str:
    """What is missing for the binding ('': nothing)."""
    if not shutil.which("g++"):
        return "g++"
    try:
        import torch
    except ImportError:
        return "torch"
    if not os.path.exists(os.path.join(os.path.dirname(torch.__file__), "include", "torch", "csrc", "autograd", "python_variable.h")):
        return "torch's headers"
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        return "Python.h"
    return ""


def build_binding(force: bool = False) -> str:
    """Builds _binding.so, the marshalling of the attention operators, against the torch that is installed."""
    lacks = binding_lacks()
    if lacks:
        sys.stderr.write(f"{os.path.basename(BINDING)} is left out: {lacks} is missing (attention.py needs it, the C ABI does not)\n")
        return ""
    if not force and not needs_build(BINDING):
        return BINDING
    import torch
    inside = os.path.dirname(torch.__file__)
    inc = [os.path.join(inside, "include"), os.path.join(inside, "include", "torch", "csrc", "api", "include"),
           sysconfig.get_paths()["include"], os.path.join(os.path.dirname(os.path.dirname(nvcc_path())), "include"), os.path.join(ROOT, "include")]
    cmd = (["g++", "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            f'-DFPSK_BINDING_MARK="{binding_mark()}"']
           + [f"-I{d}" for d in inc] + [os.path.join(HERE, "csrc", "binding.cpp"), "-L" + os.path.join(inside, "lib"), "-ltorch_python",
                                        "-ltorch_cpu", "-lc10", "-o", BINDING])
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("g++ failed")
    return BINDING


def build(verbose: bool = False, force: bool = False, bounds: bool = False) -> str:
    """Builds libfpsk.so and the binding, or with bounds=True the index-checked variant libfpsk_bounds.so."""
    out = LIB_BOUNDS if bounds else LIB
    if force or needs_build(out):
        _build_library(out, verbose, bounds)
    if not bounds:
        build_binding(force)
    return out


def _build_library(out: str, verbose: bool, bounds: bool) -> None:
    arch = ["-gencode", "arch=compute_100a,code=sm_100a"]
    flags = arch + ["-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(HERE, "csrc")]
    # extra flags, e.g. FPSK_NVCC_FLAGS=-DFPSK_MEASURE for the build that records in-kernel time stamps
    flags += os.environ.get("FPSK_NVCC_FLAGS", "").split()
    if bounds:
        flags += ["-DFPSK_DEBUG_BOUNDS"]
    if verbose:
        flags += ["-Xptxas", "-v"]

    def run(cmd):
        res = subprocess.run(cmd, capture_output=True, text=True)
        if verbose or res.returncode != 0:
            sys.stderr.write(res.stdout + res.stderr)
        if res.returncode != 0:
            raise RuntimeError("nvcc failed")

    with tempfile.TemporaryDirectory() as tmp:
        # one nvcc per source file, side by side
        objs = [os.path.join(tmp, os.path.basename(f) + ".o") for f in sources()]
        with ThreadPoolExecutor(max_workers=os.cpu_count() or 1) as pool:
            list(pool.map(lambda fo: run([nvcc_path()] + flags + ["-c", fo[0], "-o", fo[1]]), zip(sources(), objs)))
        run([nvcc_path()] + arch + ["-shared", "-Xcompiler", "-fPIC"] + objs + ["-o", out])


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv, force=True, bounds="--bounds" in sys.argv))
