"""Builds libpercache.so (the C-ABI library) in-tree with nvcc for sm_100a, and the compiled part of the Python binding.

    python -m paper_2601_11553_b200.build [--force]

The result sits next to this file; nothing is written outside the package.
"""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ_DIR = os.path.join(HERE, "_build")
LIB_PATH = os.path.join(HERE, "libpercache.so")
BINDING_PATH = os.path.join(HERE, "_ops_binding" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
SOURCES = ["percache_api.cu", "kernels_mem.cu", "kernels_ref.cu", "gemm_umma.cu", "gemm_small.cu", "attn_umma.cu", "attn_decode.cu", "attn_plan.cu", "attn_tree.cu", "attn_narrow.cu", "attn_weights.cu", "slots.cu", "ops_api.cu", "gemm_noalloc.cu", "qa_bank.cu", "wait_probe.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def _deps_mtime() -> float:
    paths = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    paths.append(os.path.join(os.path.dirname(HERE), "include", "percache.h"))
    paths.append(os.path.abspath(__file__))
    return max(os.path.getmtime(p) for p in paths)


def _current(path: str) -> bool:
    return os.path.exists(path) and os.path.getmtime(path) >= _deps_mtime()


def build_library(verbose: bool = False) -> None:
    os.makedirs(OBJ_DIR, exist_ok=True)
    nvcc = _nvcc()

    def compile_one(src: str) -> str:
        obj = os.path.join(OBJ_DIR, src.replace(".cu", ".o"))
        cmd = [nvcc, *NVCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed for {src}:\n{r.stdout}\n{r.stderr}")
        if verbose:
            sys.stderr.write(r.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = LIB_PATH + ".tmp"
    r = subprocess.run([nvcc, "-shared", "-o", tmp, *objs, "-cudart", "static"], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB_PATH)


def build_binding() -> None:
    tmp = BINDING_PATH + ".tmp"
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden", "-Wall",
           "-I" + sysconfig.get_paths()["include"], os.path.join(CSRC, "ops_binding.cpp"), "-o", tmp]
    try:
        r = subprocess.run(cmd, capture_output=True, text=True)
    except OSError as e:
        raise RuntimeError(f"{cmd[0]} failed for ops_binding.cpp: {e}") from e
    if r.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed for ops_binding.cpp:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, BINDING_PATH)


def build(force: bool = False, verbose: bool = False) -> str:
    """The library, and the binding where it can be compiled (it needs Python's headers and a host compiler, the library does not
    need it): without it the cache operators' Python functions raise, and all else works."""
    if force or not _current(LIB_PATH):
        build_library(verbose)
    if force or not _current(BINDING_PATH):
        try:
            build_binding()
        except RuntimeError as e:
            if os.path.exists(BINDING_PATH):
                os.remove(BINDING_PATH)          # older than the library's interface
            sys.stderr.write(f"warning: the Python binding of the cache operators was not built: {e}\n")
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
