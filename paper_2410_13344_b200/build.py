"""Builds libcerb.so (hand-written CUDA for sm_100a) next to this file with nvcc, and _paged.so, the native part of the binding, with g++."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libcerb.so")
SOURCES = ["api.cu", "glue.cu", "gemm_f32.cu", "gemm_bf16.cu", "gemm_tile.cu", "gemm_few.cu", "gemm_rows.cu", "attention.cu", "heads.cu", "gate_accept.cu", "launch_order.cu",
           "pages.cu", "paged_attention.cu", "page_select.cu"]
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC]


BINDING = os.path.join(HERE, "_paged.so")


def _build_binding(force: bool) -> None:
    src = os.path.join(CSRC, "paged_binding.cpp")
    if not (force or _stale(BINDING, [src, os.path.join(ROOT, "include", "cerb.h")])):
        return
    import sysconfig

    import torch
    base = os.path.join(os.path.dirname(torch.__file__), "include")
    cuda = os.path.dirname(os.path.dirname(NVCC))
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    includes = [os.path.join(ROOT, "include"), base, os.path.join(base, "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"],
                os.path.join(cuda, "include")]
    _run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI]
         + [x for i in includes for x in ("-isystem" if i != includes[0] else "-I", i)]
         + [src, "-o", BINDING, "-L", lib, "-ltorch_python", "-ltorch", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda", "-Wl,-rpath," + lib])


def _run(cmd) -> str:
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("build failed: %s\n%s\n%s" % (" ".join(cmd), r.stdout, r.stderr))
    return r.stderr


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build(verbose: bool = False, force: bool = False) -> str:
    os.makedirs(OBJ, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in sorted(os.listdir(CSRC)) if f.endswith(".cuh")]
    headers.append(os.path.join(ROOT, "include", "cerb.h"))
    jobs = []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(OBJ, src.replace(".cu", ".o"))
        if force or _stale(o, [s] + headers):
            cmd = [NVCC] + FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", s, "-o", o]
            jobs.append(cmd)

    with ThreadPoolExecutor(max_workers=min(8, len(jobs) + 1)) as ex:
        native = ex.submit(_build_binding, force)
        logs = list(ex.map(_run, jobs))
        native.result()
    if verbose:
        sys.stderr.write("\n".join(logs))
    objs = [os.path.join(OBJ, s.replace(".cu", ".o")) for s in SOURCES]
    if force or jobs or _stale(LIB, objs):
        _run([NVCC, "-shared", "-o", LIB] + objs + ["-lcudart"])
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv, force="-f" in sys.argv))
