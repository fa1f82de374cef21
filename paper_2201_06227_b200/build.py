"""Compile the CUDA library for sm_100a, in-tree (``python -m paper_2201_06227_b200.build``)."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

HERE = Path(__file__).resolve().parent
CSRC = HERE / "csrc"
LIB = HERE / "libegeria.so"
BINDING = HERE / "_ops_python.so"             # the operators' calls from Python (csrc/ops/ops_python.cpp)
BINDING_SOURCE = CSRC / "ops" / "ops_python.cpp"
LIB_CHECKED = HERE / "libegeria_checked.so"   # the same sources with -DEGERIA_CHECKED (csrc/check.cuh)
SOURCES = [CSRC / "egeria_api.cu", CSRC / "ops" / "ops_api.cu", CSRC / "ops" / "gated_api.cu", CSRC / "ops" / "muon_api.cu"]
HEADERS = [*sorted(CSRC.rglob("*.cuh")), *sorted(CSRC.rglob("*.h")), *sorted((HERE.parent / "include").glob("*.h"))]

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-shared", "-Xcompiler", "-fPIC", "-Xptxas", "-v", "-t", "0",   # -t 0: the sources side by side
]


def stale(lib: Path = LIB) -> bool:
    if not lib.exists():
        return True
    t = lib.stat().st_mtime
    return any(p.stat().st_mtime > t for p in ([BINDING_SOURCE] if lib == BINDING else SOURCES) + HEADERS)


def _compile(lib: Path, extra, verbose: bool) -> None:
    nvcc = os.environ.get("NVCC", "nvcc")
    tmp = lib.with_suffix(f".so.tmp{os.getpid()}")
    cmd = [nvcc, *NVCC_FLAGS, *extra, "-o", str(tmp), *map(str, SOURCES)]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
    if res.returncode != 0:
        raise RuntimeError(f"nvcc failed building {lib.name}")
    os.replace(tmp, lib)


def _compile_binding(verbose: bool) -> None:
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    tmp = BINDING.with_suffix(f".so.tmp{os.getpid()}")
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
           *(f"-I{p}" for p in [*cpp_extension.include_paths(), sysconfig.get_paths()["include"]]), "-o", str(tmp), str(BINDING_SOURCE),
           *(f"-L{p}" for p in cpp_extension.library_paths()), "-lc10", "-ltorch_cpu", "-ltorch", "-ltorch_python"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
    if res.returncode != 0:
        raise RuntimeError(f"building {BINDING.name} failed")
    os.replace(tmp, BINDING)


def build(force: bool = False, verbose: bool = False, checked: bool = True) -> Path:
    """Build libegeria.so and _ops_python.so (and, unless checked=False, libegeria_checked.so) if missing or
    older than the sources.  Raises on failure."""
    wanted = [(LIB, [])] + ([(LIB_CHECKED, ["-DEGERIA_CHECKED"])] if checked else [])
    with ThreadPoolExecutor() as pool:
        jobs = [pool.submit(_compile, lib, extra, verbose) for lib, extra in wanted if force or stale(lib)]
        if force or stale(BINDING):
            jobs.append(pool.submit(_compile_binding, verbose))
    for job in jobs:
        job.result()
    return LIB


if __name__ == "__main__":
    build(force="--force" in sys.argv, verbose=True)
    print(LIB)
    print(LIB_CHECKED)
    print(BINDING)
