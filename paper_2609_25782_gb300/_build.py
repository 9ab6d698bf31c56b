"""Compile libkvtier.so in-tree with nvcc for sm_103a, and with the C compiler the
module that Pool's calls per layer go through (_calls, where Python's headers are).

The translation units (SOURCES) compile in parallel and are linked with the static CUDA runtime,
so the library needs only the driver at run time.
"""
from __future__ import annotations

import os
import shlex
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libkvtier.so")
# Named for this Python: another one in the same tree builds its own and does not load it.
CALLS = os.path.join(HERE, "_calls" + sysconfig.get_config_var("EXT_SUFFIX"))
PYTHON_H = os.path.join(sysconfig.get_paths()["include"], "Python.h")
SOURCES = ["decode_kernels.cu", "turn_kernels.cu", "copy_kernels.cu", "sparse_kernels.cu",
           "attend_kernels.cu", "page_kernels.cu", "pool.cpp", "pages.cpp", "sparse.cpp", "noalloc.cu"]
HEADERS = ["kvt_internal.h", "pool_state.h", "decode_launch.h", "turn_plan.h", "tile_ops.cuh",
           "cluster.cuh", "cache_ops.h", os.path.join("..", "..", "include", "kvtier.h")]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libkvtier.so")


def calls_command(to: str) -> list[str]:
    return [*shlex.split(os.environ.get("CC") or "gcc"), "-O2", "-shared", "-fPIC", "-I", os.path.dirname(PYTHON_H),
            os.path.join(CSRC, "calls.c"), "-o", to]


def _stale() -> bool:
    made = [LIB] + ([CALLS] if os.path.exists(PYTHON_H) else [])
    if not all(os.path.exists(x) for x in made):
        return True
    t = min(os.path.getmtime(x) for x in made)
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS + ["calls.c"]] + [os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    cc = nvcc()
    out_dir = os.path.join(HERE, "_build")
    os.makedirs(out_dir, exist_ok=True)
    # KVT_EXTRA_NVCC_FLAGS: extra -D tuning definitions for experiments
    extra_flags = os.environ.get("KVT_EXTRA_NVCC_FLAGS", "").split()
    common = [cc, "-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", *ARCH,
              "-I", os.path.join(HERE, "..", "include"), *extra_flags]
    procs, objs = [], []
    for src in SOURCES:
        obj = os.path.join(out_dir, src + ".o")
        objs.append(obj)
        extra = ["-Xptxas", "-v"] if verbose and src.endswith(".cu") else []
        procs.append((src, subprocess.Popen(common + extra + ["-c", os.path.join(CSRC, src), "-o", obj],
                                            stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                                            text=True)))
    if os.path.exists(PYTHON_H):
        procs.append(("calls.c", subprocess.Popen(calls_command(CALLS + ".tmp"), stdout=subprocess.PIPE,
                                                  stderr=subprocess.STDOUT, text=True)))
    for src, p in procs:
        out, _ = p.communicate()
        if p.returncode != 0:
            raise RuntimeError(f"compiler failed on {src}:\n{out}")
        if verbose and out:
            sys.stderr.write(out)
    tmp = LIB + ".tmp"
    res = subprocess.run([cc, "-shared", *ARCH, "-o", tmp, *objs], capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed:\n{res.stdout}{res.stderr}")
    os.replace(tmp, LIB)
    if os.path.exists(PYTHON_H):
        os.replace(CALLS + ".tmp", CALLS)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
