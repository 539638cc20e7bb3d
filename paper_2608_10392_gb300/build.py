"""Builds libunif_moe.so (the C-ABI library) in-tree for sm_103a with nvcc, and
_binding.so (the Python module of its handle-free operators) with g++.

Each translation unit compiles in its own process (in parallel); the objects
link into paper_2608_10392_gb300/lib/libunif_moe.so, and _binding.so beside it
links with that library and torch's. Nothing is installed outside the repository.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIBDIR = os.path.join(HERE, "lib")
LIB = os.path.join(LIBDIR, "libunif_moe.so")
BINDING_SRC = os.path.join(CSRC, "binding.cpp")
BINDING_OBJ = os.path.join(LIBDIR, "binding.o")
BINDING = os.path.join(LIBDIR, "_binding.so")
SOURCES = ["unif_moe.cu", "route_permute.cu", "gemm_simt.cu", "gemm_tc.cu", "gemm_ws.cu",
           "backward.cu", "diagnostics.cu", "gemm_fused.cu", "gemm_pair.cu",
           "bundles.cu", "block_norm.cu", "balance.cu", "mxfp4.cu",
           "fp4_product.cu"]
HEADERS = ["internal.cuh", "decide.cuh", "items.cuh", "tc_common.cuh", "per_device.h",
           os.path.join("..", "..", "include", "unif_moe.h")]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def _binding_cmd():
    """g++ commands that compile and link the Python module, against the torch that
    this interpreter imports."""
    import torch
    root = os.path.dirname(os.path.abspath(torch.__file__))
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc())))
    inc = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
           os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    cxx = os.environ.get("CXX") or "g++"
    compile_ = [cxx, "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden"] \
        + ["-I" + i for i in inc] + ["-c", BINDING_SRC, "-o", BINDING_OBJ]
    link = [cxx, "-shared", BINDING_OBJ, "-L" + LIBDIR, "-lunif_moe", "-L" + os.path.join(root, "lib"),
            "-ltorch_python", "-ltorch", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda",
            "-Wl,-rpath,$ORIGIN"]
    return compile_, link


def build(force: bool = False, verbose: bool = False, extra_flags=()) -> str:
    os.makedirs(LIBDIR, exist_ok=True)
    headers = [os.path.join(CSRC, h) for h in HEADERS]
    objs = []
    jobs = []
    flags = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC,-fvisibility=hidden"] + list(extra_flags)
    for src in SOURCES:
        path = os.path.join(CSRC, src)
        obj = os.path.join(LIBDIR, src.replace(".cu", ".o"))
        objs.append(obj)
        if force or _stale(obj, [path] + headers):
            cmd = [nvcc()] + ARCH + flags + ["-c", path, "-o", obj]
            jobs.append(cmd)

    binding_compile, binding_link = _binding_cmd()
    if force or _stale(BINDING_OBJ, [BINDING_SRC, headers[-1]]):
        jobs.append(binding_compile)

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("build failed:\n%s\n%s%s" % (" ".join(cmd), r.stdout, r.stderr))
        if verbose:
            sys.stderr.write(r.stdout + r.stderr)
        return r

    with cf.ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        list(ex.map(run, jobs))
    if force or jobs or _stale(LIB, objs):
        tmp = LIB + ".tmp%d" % os.getpid()
        run([nvcc()] + ARCH + ["-shared", "-o", tmp] + objs)
        os.replace(tmp, LIB)
    if force or _stale(BINDING, [BINDING_OBJ, LIB]):
        tmp = BINDING + ".tmp%d" % os.getpid()
        run(binding_link + ["-o", tmp])
        os.replace(tmp, BINDING)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
