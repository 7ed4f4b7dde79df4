"""Build of the in-tree CUDA library ``libmisat.so`` (sm_103a) with nvcc.

Each translation unit is compiled in parallel with
``-gencode arch=compute_103a,code=sm_103a -lineinfo`` and linked against the shared
CUDA runtime, so the library and PyTorch use one runtime instance.  The calls of the KV
operators on torch tensors (``_calls.so``, C++) are built beside it, where PyTorch, g++ and Python's
headers are there; the library needs none of them.
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
CALLS_FOR = os.path.join(BUILD, "calls_for.txt")
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


def _older(target, sources) -> bool:
    deps = [os.path.join(CSRC, f) for f in sources] + [os.path.join(ROOT, "include", "misat.h")]
    return not os.path.exists(target) or any(os.path.getmtime(d) > os.path.getmtime(target) for d in deps)


def _stale() -> bool:
    return _older(LIB, SOURCES + HEADERS)


def _torch_home() -> str:
    spec = importlib.util.find_spec("torch")  # (importing it takes far longer than compiling)
    if spec is None or not spec.origin:
        raise RuntimeError("PyTorch not found: the calls on torch tensors cannot be built")
    return os.path.dirname(spec.origin)


def _calls_need() -> str:
    """What the calls on torch tensors need and is not there, or an empty text."""
    try:
        home = _torch_home()
    except RuntimeError:
        return "PyTorch"
    if not os.path.exists(os.path.join(home, "lib", "libtorch_cuda.so")):
        return "PyTorch with CUDA"
    if shutil.which("g++") is None:
        return "g++"
    return "" if os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")) else "Python's headers"


def _calls_for() -> str:
    """The Python and the PyTorch that the calls are built for."""
    home = _torch_home()
    with open(os.path.join(home, "version.py")) as f:
        return "\n".join((sys.version, home, f.read()))


def _calls_stale() -> bool:
    if _older(CALLS, [CALLS_SOURCE]) or not os.path.exists(CALLS_FOR):
        return True
    with open(CALLS_FOR) as f:
        return f.read() != _calls_for()


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
          "-ltorch_cpu", "-lc10_cuda", "-lc10", "-L", os.path.dirname(LIB), "-l:" + os.path.basename(LIB),
          "-L", os.path.join(cuda, "lib64"), "-lcudart", "-Wl,-rpath,$ORIGIN"], "link of the calls on torch tensors")
    os.replace(tmp, CALLS)
    with open(CALLS_FOR, "w") as f:
        f.write(_calls_for())


def build(force: bool = False, verbose: bool = False, extra_flags=()) -> str:
    lib, need = force or _stale(), _calls_need()
    calls = not need and (force or _calls_stale())
    if need and (lib or not os.path.exists(CALLS)):
        print(f"{need} not found: the library is built without the calls on torch tensors", file=sys.stderr)
        if os.path.exists(CALLS):
            os.remove(CALLS)  # made for another library
    if not lib and not calls:
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
        calls_obj = ex.submit(_compile_calls) if calls else None
        objs = list(ex.map(compile_one, SOURCES)) if lib else []
    if lib:
        tmp = LIB + f".tmp{os.getpid()}"
        cmd = [cc, *ARCH, "-shared", "-cudart", "shared", "-o", tmp, *objs]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
        os.replace(tmp, LIB)
    if calls:
        _link_calls(calls_obj.result())  # (an error in them leaves the library in its place)
    return LIB


if __name__ == "__main__":
    build(force="--force" in sys.argv, verbose="--verbose" in sys.argv,
          extra_flags=["-Xptxas", "-v"] if "--ptxas" in sys.argv else [])
    print(LIB)
