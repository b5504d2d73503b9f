"""Builds libbuddy.so in-tree with nvcc for sm_103a (no cmake, no torch), and _calls.so,
which turns tensors into its arguments, with the host compiler and torch's headers."""
from __future__ import annotations

import concurrent.futures as cf
import importlib.metadata
import os
import shutil
import subprocess
import sys
import sysconfig
from importlib.util import find_spec

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT_DIR = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libbuddy.so")
SOURCES = ["api.cu", "kernels.cu", "attention.cu", "gemm_simt.cu", "gemm_tc.cu", "noalloc.cu", "gemm_pf.cu",
           "attn_pf.cu", "prefill.cu", "attn_cl.cu", "pages.cu", "kv4_rows.cu", "kv4_attn.cu", "kv4_pf.cu", "kv4_pages.cu", "kv4_lists.cu"]
CALLS = os.path.join(HERE, "_calls.so")
CALLS_FOR = os.path.join(OUT_DIR, "calls_for.txt")   # the torch and the command that it was built with
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
         "--expt-relaxed-constexpr", "-Xptxas", "-warn-spills"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _stale(obj: str, src: str) -> bool:
    if not os.path.exists(obj):
        return True
    deps = [src] + [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    deps.append(os.path.join(HERE, "..", "include", "buddy.h"))
    t = os.path.getmtime(obj)
    return any(os.path.getmtime(d) > t for d in deps)


def _calls_command(nvcc: str) -> list:
    torch = os.path.dirname(find_spec("torch").origin)
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
            "-I" + sysconfig.get_paths()["include"], "-isystem", os.path.join(torch, "include"), "-isystem", cuda,
            os.path.join(CSRC, "calls.cpp"), "-o", CALLS + ".tmp", "-L" + os.path.join(torch, "lib"),
            "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda"]


def _torch_version() -> str:
    try:
        return importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:
        return ""


def _calls_built_for() -> str:
    try:
        return open(CALLS_FOR).read()
    except FileNotFoundError:
        return ""


def build(verbose: bool = False, force: bool = False) -> str:
    nvcc = _nvcc()
    os.makedirs(OUT_DIR, exist_ok=True)
    objs = []
    jobs = []
    for s in SOURCES:
        src = os.path.join(CSRC, s)
        obj = os.path.join(OUT_DIR, s.replace(".cu", ".o"))
        objs.append(obj)
        if force or _stale(obj, src):
            jobs.append([nvcc, *ARCH, *FLAGS, "-c", src, "-o", obj])
    kernels = bool(jobs)
    calls_command = _calls_command(nvcc)
    calls_for = _torch_version() + "\n" + " ".join(calls_command)
    calls = force or _stale(CALLS, os.path.join(CSRC, "calls.cpp")) or _calls_built_for() != calls_for
    if calls:
        jobs.append(calls_command)
    with cf.ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        results = list(ex.map(lambda cmd: subprocess.run(cmd, capture_output=True, text=True), jobs))
    for cmd, r in zip(jobs, results):
        if verbose or r.returncode != 0:
            sys.stderr.write(r.stdout + r.stderr)
        if r.returncode != 0:
            raise RuntimeError(f"failed: {' '.join(cmd)}")
    if calls:
        os.replace(CALLS + ".tmp", CALLS)
        with open(CALLS_FOR, "w") as f:
            f.write(calls_for)
    if kernels or not os.path.exists(LIB):
        link = [nvcc, *ARCH, "-shared", "-o", LIB + ".tmp", *objs]
        r = subprocess.run(link, capture_output=True, text=True)
        if r.returncode != 0:
            sys.stderr.write(r.stdout + r.stderr)
            raise RuntimeError("link failed")
        os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv, force="-f" in sys.argv))
