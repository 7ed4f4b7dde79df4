"""Build of the in-tree CUDA library ``libmisat.so`` (sm_103a) with nvcc.

Each translation unit is compiled in parallel with
``-gencode arch=compute_103a,code=sm_103a -lineinfo`` and linked against the shared
CUDA runtime, so the library and PyTorch use one runtime instance.  The calls of the KV
operators on torch tensors (``_calls.so``, C++) are built beside it.
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
LIB = os.path.join(HERE, "libmisat.so")
CALLS = os.path.join(HERE, "_calls.so")
CALLS_SOURCE = "torch_calls.cpp"
SOURCES = ["api.cu", "hash.cu", "probe.cu", "route.cu", "select.cu", "commit.cu", "evict.cu", "gindex.cu",
           "overload.cu", "stage.cu", "rotary.cu", "kv.cu", "attend.cu"]
HEADERS = ["common.cuh", "gindex.cuh", "kernels.h", "tick_scale.h", "kv.h", "runs.cuh", "tensor.cuh"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def nvcc() -> str:
    p = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(p):
        raise RuntimeError("nvcc not found: the MISA-T CUDA library cannot be built")
    return p


def _flags(extra=()):
    return ["-O3", "-std=c++17", *ARCH, "-lineinfo", "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr",
            "-I", os.path.join(ROOT, "include"), *extra]


def _stale() -> bool:
    if not (os.path.exists(LIB) and os.path.exists(CALLS)):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(CALLS))
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS + [CALLS_SOURCE]]
    deps.append(os.path.join(ROOT, "include", "misat.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def _torch_home() -> str:
    spec = importlib.util.find_spec("torch")  # (importing it takes far longer than compiling)
    if spec is None or not spec.origin:
        raise RuntimeError("PyTorch not found: the calls on torch tensors cannot be built")
    return os.path.dirname(spec.origin)


def _run(cmd, what):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what} failed:\n{r.stdout}\n{r.stderr}")
    return r


def _compile_calls() -> str:
    torch_include = os.path.join(_torch_home(), "include")
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc())))
    obj = os.path.join(BUILD, "torch_calls.o")
    _run(["g++", "-O2", "-std=c++17", "-fPIC", "-I", torch_include,
          "-I", os.path.join(torch_include, "torch", "csrc", "api", "include"),
          "-I", sysconfig.get_paths()["include"], "-I", os.path.join(cuda, "include"),
          "-c", os.path.join(CSRC, CALLS_SOURCE), "-o", obj], f"g++ on {CALLS_SOURCE}")
    return obj


def _link_calls(obj) -> None:
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc())))
    tmp = CALLS + f".tmp{os.getpid()}"
    _run(["g++", "-shared", "-o", tmp, obj, "-L", os.path.join(_torch_home(), "lib"), "-ltorch_python", "-ltorch_cuda",
          "-ltorch_cpu", "-lc10_cuda", "-lc10", "-L", HERE, "-l:" + os.path.basename(LIB),
          "-L", os.path.join(cuda, "lib64"), "-lcudart", "-Wl,-rpath,$ORIGIN"], "link of the calls on torch tensors")
    os.replace(tmp, CALLS)


def build(force: bool = False, verbose: bool = False, extra_flags=()) -> str:
    if not force and not _stale():
        return LIB
    os.makedirs(BUILD, exist_ok=True)
    cc = nvcc()

    def compile_one(src):
        obj = os.path.join(BUILD, src.replace(".cu", ".o"))
        cmd = [cc, *_flags(extra_flags), "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), file=sys.stderr)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
        if verbose and r.stderr:
            print(r.stderr, file=sys.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        calls = ex.submit(_compile_calls)
        objs = list(ex.map(compile_one, SOURCES))
        calls_obj = calls.result()
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [cc, *ARCH, "-shared", "-cudart", "shared", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    _link_calls(calls_obj)
    return LIB


if __name__ == "__main__":
    build(force="--force" in sys.argv, verbose="--verbose" in sys.argv,
          extra_flags=["-Xptxas", "-v"] if "--ptxas" in sys.argv else [])
    print(LIB)
