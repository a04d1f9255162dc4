"""Build ``libecho.so`` in-tree with nvcc for sm_103a (GB300).

The translation units compile in parallel and link into one shared library
exporting the C ABI of ``include/echo.h``.  The overlap test compiles once per
variant family (launch interval x proportional model), four objects in parallel.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libecho.so")
BUILD_DIR = os.path.join(PKG, "_build")
# (source, extra nvcc flags, object)
UNITS = [(f, [], f + ".o") for f in ("echo_kernels.cu", "echo_compose.cu", "echo_levels.cu", "echo_dataflow.cu", "echo_host.cpp",
                                        "echo_ops.cpp", "echo_ops_embed.cu", "echo_ops_norm.cu", "echo_ops_ortho.cu")] + [
    ("echo_overlap.cu", [f"-DECHO_OV_LAUNCH={l}", f"-DECHO_OV_PROP={p}"], f"echo_overlap_l{l}_p{p}.o")
    for l in (0, 1) for p in (0, 1)]
SOURCES = sorted({u[0] for u in UNITS})
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libecho.so")
    return exe


def _flags():
    return ARCH + ["-O3", "-lineinfo", "-std=c++17", "-I", INCLUDE, "-I", CSRC,
                   "-Xcompiler", "-fPIC,-ffp-contract=off,-fno-fast-math", "--expt-relaxed-constexpr"]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(INCLUDE, "echo.h"),
                                                                 os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False, ptxas_info: bool = False) -> str:
    if not force and not _stale():
        return LIB
    os.makedirs(BUILD_DIR, exist_ok=True)
    exe = nvcc()

    def compile_one(unit):
        src, extra, obj_name = unit
        obj = os.path.join(BUILD_DIR, obj_name)
        cmd = [exe] + _flags() + extra + (["-Xptxas", "-v"] if ptxas_info and src.endswith(".cu") else []) + \
            ["-c", os.path.join(CSRC, src), "-o", obj]
        if src.endswith(".cpp"):
            cmd[1:1] = ["-x", "cu"]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
        if verbose or ptxas_info:
            sys.stderr.write(r.stdout + r.stderr)
        return obj

    with ThreadPoolExecutor(len(UNITS)) as ex:
        objs = list(ex.map(compile_one, UNITS))
    tmp = LIB + f".{os.getpid()}.tmp"
    r = subprocess.run([exe] + ARCH + ["-shared", "-o", tmp] + objs, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True, ptxas_info="--ptxas" in sys.argv))
