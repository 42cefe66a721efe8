"""Build the CUDA library in-tree: ``python -m paper_2609_19758_b200.build``.

Compiles every ``csrc/*.cu`` for sm_100a with nvcc into ``libfpsk.so`` next to this file, and ``csrc/binding.cpp`` with g++ into
the Python module ``_binding.so``.
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


def needs_build(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    if lib == BINDING:
        return any(os.path.getmtime(d) > t for d in [os.path.join(HERE, "csrc", "binding.cpp"), os.path.join(ROOT, "include", "fpsk_attention.h")])
    deps = sources() + glob.glob(os.path.join(HERE, "csrc", "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def build_binding(force: bool = False) -> str:
    """Builds _binding.so, the marshalling of the attention operators, against the torch that is installed."""
    if not force and not needs_build(BINDING):
        return BINDING
    import torch
    inside = os.path.dirname(torch.__file__)
    inc = [os.path.join(inside, "include"), os.path.join(inside, "include", "torch", "csrc", "api", "include"),
           sysconfig.get_paths()["include"], os.path.join(os.path.dirname(os.path.dirname(nvcc_path())), "include"), os.path.join(ROOT, "include")]
    cmd = (["g++", "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
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
    if not bounds:
        build_binding(force)
    if not force and not needs_build(out):
        return out
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
    return out


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv, force=True, bounds="--bounds" in sys.argv))
