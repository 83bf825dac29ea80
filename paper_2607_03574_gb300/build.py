"""Build the NDVM C-ABI library (libndvm.so) in-tree with nvcc for sm_103a.

Translation units compile in parallel; the result is linked as one shared
library with the CUDA runtime linked statically.  Where PyTorch is installed, a Python
module on top of it (ndvm_torch.so) holds the network operators' autograd nodes; the
library does not need it.  Run ``python -m paper_2607_03574_gb300.build`` or call
:func:`build`.
"""
from __future__ import annotations

import concurrent.futures as cf
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
OUT_DIR = os.path.join(HERE, "_build")
LIB = os.path.join(OUT_DIR, "libndvm.so")
TORCH_OPS = os.path.join(OUT_DIR, "ndvm_torch.so")  # the network operators' autograd nodes (a Python module)
TORCH_OPS_SOURCE = os.path.join(CSRC, "net", "torch_ops.cpp")

SOURCES = ["tape.cpp", "trace_scheme.cpp", "trace_bytecode.cpp", "plan.cpp", "compact.cpp", "capi.cpp", "replay.cu", "scalar.cu", "matrix.cu",
           "net/netapi.cpp", "net/norm.cu", "net/dropout.cu", "net/gated.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def _nvcc() -> str:
    for c in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("nvcc not found: the NDVM library needs the CUDA toolkit to build")


def _newer(target: str, files: list[str]) -> bool:
    """Whether the target is missing or one of the files (or this one) was changed after it was made."""
    return not os.path.exists(target) or any(os.path.getmtime(f) > os.path.getmtime(target) for f in (*files, os.path.abspath(__file__)))


def _stale() -> bool:
    files = [os.path.join(d, f) for d in (CSRC, os.path.join(CSRC, "net")) for f in os.listdir(d)]
    files.remove(TORCH_OPS_SOURCE)
    return _newer(LIB, [*files, os.path.join(INCLUDE, "ndvm.h")])


def _torch_ops_stale() -> bool:
    try:
        with open(_torch_ops_record()) as f:
            same = f.read() == _built_against()
    except OSError:
        same = False
    return not same or _newer(TORCH_OPS, [TORCH_OPS_SOURCE, os.path.join(INCLUDE, "ndvm.h")])


def _torch_root() -> str | None:
    spec = importlib.util.find_spec("torch")  # (not imported: that takes longer than finding it)
    return list(spec.submodule_search_locations)[0] if spec else None


def _torch_ops_record() -> str:
    return TORCH_OPS + ".for"


def _built_against() -> str:
    """The Python and the PyTorch (its place and its version file) that the module fits: another one's binary
    interface is another."""
    root = _torch_root()
    try:
        with open(os.path.join(root or "", "version.py")) as f:
            version = f.read()
    except OSError:
        version = ""
    return f"{sys.implementation.cache_tag}\n{root}\n{version}"


def _compile_torch_ops() -> str:
    root, cuda = _torch_root(), os.path.dirname(os.path.dirname(_nvcc()))
    if root is None:
        raise RuntimeError("PyTorch not found: the network operators are built against it")
    obj = os.path.join(OUT_DIR, "net_torch_ops.cpp.o")
    include = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
               sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", *("-I" + d for d in include), "-c",
           TORCH_OPS_SOURCE, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compiling net/torch_ops.cpp failed:\n{r.stdout}\n{r.stderr}")
    return obj


def _link_torch_ops(obj: str) -> None:
    lib = os.path.join(_torch_root(), "lib")
    tmp = TORCH_OPS + f".tmp{os.getpid()}"
    cmd = ["g++", "-shared", "-o", tmp, obj, "-L" + lib, "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-ltorch_python",
           "-L" + OUT_DIR, "-l:libndvm.so", "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"linking ndvm_torch.so failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, TORCH_OPS)
    with open(_torch_ops_record(), "w") as f:
        f.write(_built_against())


def build(force: bool = False, verbose: bool = False, torch_ops: bool | None = None) -> str:
    """Makes what is missing or out of date.  torch_ops: the autograd nodes' module too (None: where PyTorch is
    installed); the library is made first and stands without it."""
    library = force or _stale()
    module = (_torch_root() is not None if torch_ops is None else torch_ops) and (force or _torch_ops_stale())
    if not library and not module:
        return LIB
    os.makedirs(OUT_DIR, exist_ok=True)
    nvcc = _nvcc()
    common = ["-O3", "-std=c++17", "-Xcompiler", "-fPIC", "-I" + INCLUDE, "-I" + CSRC]

    def compile_one(src: str) -> str:
        obj = os.path.join(OUT_DIR, src.replace("/", "_") + ".o")
        cmd = [nvcc, *common, "-c", os.path.join(CSRC, src), "-o", obj]
        if src.endswith(".cu"):
            cmd[1:1] = [*ARCH, "-lineinfo"]
        else:
            cmd[1:1] = ["-x", "c++"]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"compiling {src} failed:\n{r.stdout}\n{r.stderr}")
        if verbose and (r.stdout or r.stderr):
            print(r.stdout, r.stderr, file=sys.stderr)
        return obj

    with cf.ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        torch_obj = ex.submit(_compile_torch_ops) if module else None
        if library:
            objs = list(ex.map(compile_one, SOURCES))
            tmp = LIB + f".tmp{os.getpid()}"
            cmd = [nvcc, *ARCH, "-shared", "-o", tmp, *objs, "-cudart", "static"]
            r = subprocess.run(cmd, capture_output=True, text=True)
            if r.returncode != 0:
                raise RuntimeError(f"linking libndvm.so failed:\n{r.stdout}\n{r.stderr}")
            os.replace(tmp, LIB)
        if module:
            _link_torch_ops(torch_obj.result())
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
