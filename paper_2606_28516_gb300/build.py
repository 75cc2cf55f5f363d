"""Builds libclearmoe.so in-tree for sm_103a with nvcc (one process per translation unit), and the binding's compiled
part, _calls.so, with the host compiler."""
from __future__ import annotations

import concurrent.futures as cf
import os
import pathlib
import shutil
import subprocess
import sysconfig

PKG = pathlib.Path(__file__).resolve().parent
CSRC = PKG / "csrc"
OUT = PKG / "libclearmoe.so"
CALLS = PKG / "_calls.so"
BUILD = PKG / "_build"
SOURCES = ("api.cu", "route.cu", "simt.cu", "tc_gemm.cu", "tc_gemm2.cu", "noalloc.cu", "fold.cu",
           "fp8.cu", "fp8_gemm.cu", "fp8_gemm2.cu", "fp8_few.cu", "few.cu")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr"]


def nvcc() -> str:
    cand = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(cand):
        raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libclearmoe.so")
    return cand


def _compile(src: pathlib.Path, verbose: bool) -> pathlib.Path:
    obj = BUILD / (src.stem + ".o")
    cmd = [nvcc(), *ARCH, *FLAGS, "-I", str(PKG.parent / "include"), "-c", str(src), "-o", str(obj)]
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc failed on {src.name}:\n{r.stdout}\n{r.stderr}")
    if verbose and r.stderr:
        print(r.stderr)
    return obj


def build_calls(force: bool = False) -> pathlib.Path:
    """csrc/calls.c against the running interpreter's headers."""
    src, header = CSRC / "calls.c", PKG.parent / "include" / "clearmoe.h"
    if CALLS.exists() and not force and all(CALLS.stat().st_mtime >= p.stat().st_mtime for p in (src, header)):
        return CALLS
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        raise RuntimeError("no C compiler found for the binding")
    tmp = CALLS.with_suffix(".so.tmp")
    r = subprocess.run([cc, "-std=c11", "-O2", "-fPIC", "-shared", "-I", sysconfig.get_paths()["include"], "-I", str(header.parent),
                        "-o", str(tmp), str(src)], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{cc} failed on calls.c:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, CALLS)
    return CALLS


def build(verbose: bool = False, force: bool = False) -> pathlib.Path:
    build_calls(force)
    srcs = [CSRC / s for s in SOURCES]
    deps = srcs + [*CSRC.glob("*.cuh"), *CSRC.glob("*.h"), PKG.parent / "include" / "clearmoe.h"]
    if OUT.exists() and not force and all(OUT.stat().st_mtime >= p.stat().st_mtime for p in deps):
        return OUT
    BUILD.mkdir(exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=len(srcs)) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose), srcs))
    tmp = OUT.with_suffix(".so.tmp")
    cmd = [nvcc(), *ARCH, "-shared", "-o", str(tmp), *map(str, objs), "-lcudart",
           "-Xlinker", "-rpath", "-Xlinker", "/usr/local/cuda/lib64"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, OUT)
    return OUT


if __name__ == "__main__":
    import sys

    print(build(verbose="-v" in sys.argv, force=True))
