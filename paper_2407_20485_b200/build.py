"""Builds ``liba2sf.so`` in-tree with nvcc for sm_100a (cross-compiles without a GPU).

    python -m paper_2407_20485_b200.build [--force] [--verbose] [--debug]

``--debug`` builds ``liba2sf_debug.so`` from the same sources with ``-DA2SF_DEBUG``: every index
that addresses memory inside a kernel is range-checked and reported (``a2sf_debug_violations``)
instead of used.  Select it at run time with ``A2SF_LIBRARY=debug`` (see ``binding.py``).
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

PKG = Path(__file__).resolve().parent
CSRC = PKG / "csrc"
INCLUDE = PKG.parent / "include"
OBJ_DIR = PKG / "_build"
LIB_PATH = PKG / "liba2sf.so"
CALLS_SRC = CSRC / "torch_calls.cpp"
DEBUG_OBJ_DIR = PKG / "_build_debug"
DEBUG_LIB_PATH = PKG / "liba2sf_debug.so"

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC",
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (cand == "nvcc" or Path(cand).exists()):
            return cand
    raise RuntimeError("nvcc not found")


def _sources():
    return sorted(CSRC.glob("*.cu"))


def _deps_mtime() -> float:
    files = list(CSRC.glob("*.cuh")) + list(CSRC.glob("*.h")) + list(INCLUDE.glob("*.h"))
    return max(f.stat().st_mtime for f in files)


def calls_path() -> Path:
    """The Python extension that marshals torch tensors: made for one interpreter and one torch, and named after them."""
    import torch

    return PKG / f"_torch_calls.{sys.implementation.cache_tag}.torch-{torch.__version__}.so"


def missing_for_calls() -> str | None:
    """What this machine lacks to build the extension (the library itself needs nvcc alone), or None."""
    import sysconfig

    try:
        import torch
    except ImportError:
        return "torch"
    for header in (Path(torch.__file__).resolve().parent / "include/ATen/ATen.h", Path(sysconfig.get_paths()["include"]) / "Python.h"):
        if not header.exists():
            return str(header)
    return None


def build_calls(force: bool = False) -> Path:
    """Compile the extension of ``calls_path()`` (host code only)."""
    path = calls_path()
    newest = max(CALLS_SRC.stat().st_mtime, *(f.stat().st_mtime for f in INCLUDE.glob("*.h")))
    if not force and path.exists() and path.stat().st_mtime >= newest:
        return path
    import sysconfig

    import torch

    root = Path(torch.__file__).resolve().parent
    cuda = Path(_nvcc()).resolve().parent.parent / "include"
    tmp = path.with_suffix(f".tmp{os.getpid()}.so")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-o", str(tmp), str(CALLS_SRC),
           *(f"-I{p}" for p in (root / "include", root / "include/torch/csrc/api/include", cuda, sysconfig.get_paths()["include"])),
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           f"-L{root / 'lib'}", "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, path)
    return path


def build(force: bool = False, verbose: bool = False, debug: bool = False) -> Path:
    """Compile every ``csrc/*.cu`` and link the shared library (the bounds-checked one with
    ``debug``), and the extension for torch tensors where there is a torch.  Returns the library's path."""
    obj_dir, lib_path = (DEBUG_OBJ_DIR, DEBUG_LIB_PATH) if debug else (OBJ_DIR, LIB_PATH)
    extra = ["-DA2SF_DEBUG"] if debug else []
    obj_dir.mkdir(exist_ok=True)
    nvcc = _nvcc()
    hdr_m = _deps_mtime()
    jobs = []
    for src in _sources():
        obj = obj_dir / (src.stem + ".o")
        if force or not obj.exists() or obj.stat().st_mtime < max(src.stat().st_mtime, hdr_m):
            cmd = [nvcc, *NVCC_FLAGS, *extra, "-I", str(INCLUDE), "-c", str(src), "-o", str(obj)]
            if verbose:
                cmd[1:1] = ["-Xptxas", "-v"]
            jobs.append(cmd)

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
        return r.stderr

    with ThreadPoolExecutor(max_workers=min(8, max(1, len(jobs)))) as ex:
        for log in ex.map(run, jobs):
            if verbose and log:
                print(log, file=sys.stderr)
    objs = [obj_dir / (s.stem + ".o") for s in _sources()]
    if force or jobs or not lib_path.exists():
        tmp = lib_path.with_suffix(f".tmp{os.getpid()}.so")
        cmd = [nvcc, "-shared", "-gencode", "arch=compute_100a,code=sm_100a",
               "-o", str(tmp), *map(str, objs), "-cudart", "static"]
        run(cmd)
        os.replace(tmp, lib_path)
    missing = missing_for_calls()
    if missing is None:
        build_calls(force)
    else:
        print(f"{missing} is missing: built {lib_path.name} without the extension for torch tensors", file=sys.stderr)
    return lib_path


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv, debug="--debug" in sys.argv))
