"""Builds libstom_oqm.so (sm_100a only) next to this file with nvcc, and _stom_bind.so, the Python binding of the
calls that are made once per token, with g++ against the headers of the torch that is installed.  Without the binding the
library is complete but for those calls; it is built first.

    python -m paper_2510_18269_b200.build [--force] [--verbose]

nvcc cross-compiles without a GPU.  The library is kept in-tree so that it
travels with the source tree; nothing is installed into site-packages.
"""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

PKG = Path(__file__).resolve().parent
CSRC = PKG / "csrc"
INCLUDE = PKG.parent / "include"
OBJ = PKG / "_build"
LIB = PKG / "libstom_oqm.so"
BIND = PKG / "_stom_bind.so"
BUILT_FOR = OBJ / "stom_bind.txt"   # the Python and the torch that the binding was built for

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-I", str(INCLUDE), "-I", str(CSRC),
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (cand == "nvcc" or Path(cand).exists()):
            return cand
    raise RuntimeError("nvcc not found")


def sources():
    return sorted(CSRC.glob("*.cu"))


def _newer(target: Path, *patterns: str) -> bool:
    """Whether a target is there and no older than its sources of these kinds, the headers and this file."""
    files = [f for p in patterns for f in CSRC.glob(p)] + list(INCLUDE.glob("*.h")) + [Path(__file__)]
    return target.exists() and target.stat().st_mtime >= max(f.stat().st_mtime for f in files)


def _installed() -> str:
    import torch

    return f"{sys.implementation.cache_tag} torch {torch.__version__} {torch.__file__}"


def _binding_fits() -> bool:
    return _newer(BIND, "*.cpp") and BUILT_FOR.exists() and BUILT_FOR.read_text() == _installed()


def _build_binding() -> None:
    import torch

    at = Path(torch.__file__).parent
    cuda = Path(_nvcc()).parent.parent if "/" in _nvcc() else Path("/usr/local/cuda")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-I", sysconfig.get_paths()["include"], "-I", str(at / "include"), "-I",
           str(at / "include/torch/csrc/api/include"), "-I", str(cuda / "include"), "-I", str(INCLUDE),
           str(CSRC / "stom_bind.cpp"), "-o", str(BIND), "-L", str(at / "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10",
           "-lc10_cuda", f"-Wl,-rpath,{at / 'lib'}"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode:
        raise RuntimeError(f"g++ failed for stom_bind.cpp:\n{r.stdout}\n{r.stderr}")
    BUILT_FOR.write_text(_installed())


def _build_library(verbose: bool) -> None:
    nvcc = _nvcc()
    extra = ["-Xptxas", "-v"] if verbose else []

    def compile_one(src: Path) -> Path:
        obj = OBJ / (src.stem + ".o")
        cmd = [nvcc, *NVCC_FLAGS, *extra, "-c", str(src), "-o", str(obj)]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if verbose:
            sys.stderr.write(r.stderr)
        if r.returncode:
            raise RuntimeError(f"nvcc failed for {src.name}:\n{r.stdout}\n{r.stderr}")
        return obj

    with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as ex:
        objs = list(ex.map(compile_one, sources()))
    link = [nvcc, "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-o", str(LIB), *map(str, objs)]
    r = subprocess.run(link, capture_output=True, text=True)
    if r.returncode:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")


def build(force: bool = False, verbose: bool = False) -> Path:
    OBJ.mkdir(exist_ok=True)
    with ThreadPoolExecutor(max_workers=1) as ex:
        binding = ex.submit(lambda: None if not force and _binding_fits() else _build_binding())
        if force or not _newer(LIB, "*.cu", "*.cuh"):
            _build_library(verbose)
        binding.result()   # what went wrong with the binding is raised when the library is there
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
