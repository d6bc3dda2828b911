"""Build the in-tree CUDA library ``libmoe.so`` (sm_103a) with nvcc.

Each translation unit under ``csrc/`` is compiled in parallel to an object file
(``-gencode arch=compute_103a,code=sm_103a``), then linked into a shared library
next to this file. Rebuilds only what changed (source or header newer than object).
Beside it the binding's argument checks (``csrc/marshal.cpp``, host C++ on torch's headers) become
``_marshal.so``, without which the binding makes the same checks in Python.
"""
from __future__ import annotations

import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libmoe.so")
SOURCES = ["route.cu", "dispatch.cu", "gemm_f32.cu", "gemm_tc.cu", "train.cu", "norm.cu", "gate.cu",
           "ckpt.cu", "embed.cu", "vocab.cu", "orth.cu", "moe_abi.cu"]
HEADERS = ["dense_tc.cuh", "device_state.h", "moe_common.cuh", "moe_internal.h", "span.cuh", "tc_ptx.cuh"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-Xcompiler", "-O2",
         "--expt-relaxed-constexpr", "-I" + os.path.join(ROOT, "include")]


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA library cannot be built")


MARSHAL_SRC, MARSHAL = os.path.join(CSRC, "marshal.cpp"), os.path.join(HERE, "_marshal.so")


def _marshal_cmd():
    """The command that builds _marshal.so; None without torch or a host compiler."""
    spec, cxx = importlib.util.find_spec("torch"), os.environ.get("CXX") or shutil.which("g++") or shutil.which("c++")
    if spec is None or not spec.origin or not cxx:
        return None
    torch = os.path.dirname(spec.origin)
    inc = [os.path.join(torch, "include"), os.path.join(torch, "include", "torch", "csrc", "api", "include"),
           sysconfig.get_paths()["include"]]
    return [cxx, "-O2", "-std=c++17", "-fPIC", "-shared", *["-I" + i for i in inc], "-L" + os.path.join(torch, "lib"), MARSHAL_SRC,
            "-o", MARSHAL, "-ltorch_python", "-ltorch_cpu", "-lc10"]


def _stale(obj: str, src: str) -> bool:
    if not os.path.exists(obj):
        return True
    t = os.path.getmtime(obj)
    deps = [src] + [os.path.join(CSRC, h) for h in HEADERS] + [os.path.join(ROOT, "include", "moe.h")]
    return any(os.path.getmtime(p) > t for p in deps)


def build(verbose: bool = False, extra: list[str] | None = None) -> str:
    """Compile and link libmoe.so; returns its path. Raises on compiler errors."""
    os.makedirs(BUILD, exist_ok=True)
    cc = nvcc()
    extra = list(extra or [])
    jobs = []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(BUILD, src.replace(".cu", ".o"))
        if _stale(o, s) or extra:
            jobs.append([cc, *ARCH, *FLAGS, *extra, "-c", s, "-o", o])

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        return cmd, r

    marshal = None
    if not os.path.exists(MARSHAL) or os.path.getmtime(MARSHAL_SRC) > os.path.getmtime(MARSHAL):
        marshal = _marshal_cmd()
    with ThreadPoolExecutor(max_workers=min(len(SOURCES) + 1, os.cpu_count() or 4)) as ex:
        aside = ex.submit(run, marshal) if marshal else None
        for cmd, r in ex.map(run, jobs):
            if verbose or r.returncode:
                sys.stderr.write(" ".join(cmd[-3:]) + "\n" + r.stdout + r.stderr)
            if r.returncode:
                raise RuntimeError(f"nvcc failed on {cmd[-3]}")
        if aside is not None and aside.result()[1].returncode:
            sys.stderr.write("_marshal.so was not built (the binding checks its arguments in Python):\n" + aside.result()[1].stderr[-2000:])
    objs = [os.path.join(BUILD, s.replace(".cu", ".o")) for s in SOURCES]
    if jobs or not os.path.exists(LIB):
        cmd = [cc, *ARCH, "-shared", "-o", LIB, *objs, "-cudart=static"]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode:
            sys.stderr.write(r.stdout + r.stderr)
            raise RuntimeError("link of libmoe.so failed")
    return LIB


if __name__ == "__main__":
    build(verbose="-v" in sys.argv, extra=[a for a in sys.argv[1:] if a != "-v"])
    print(LIB)
