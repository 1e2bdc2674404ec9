"""Builds ``libgelo.so`` (sm_100a only) from ``csrc/*.cu`` with nvcc, in-tree, and ``_marshal.so``, which hands torch tensors to it, from
``csrc/marshal.cpp`` with the host compiler.  The library needs nvcc alone; where Python's, torch's or CUDA's headers are missing, ``_marshal.so`` is
left out with a message, and the calls of the binding that go through it raise.

    python -m paper_2603_05035_b200.build [--force]
"""
from __future__ import annotations

import concurrent.futures
import glob
import importlib.metadata
import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libgelo.so")
MARSHAL = os.path.join(HERE, "_marshal.so")
MARSHAL_FOR = os.path.join(OBJ, "marshal.for")                # the Python and torch that _marshal.so was built for

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr",
]


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every kernel source for sm_100a and link the shared library.  Returns its path."""
    os.makedirs(OBJ, exist_ok=True)
    sources = sorted(glob.glob(os.path.join(CSRC, "*.cu")))
    headers = sorted(glob.glob(os.path.join(CSRC, "*.cuh"))) + [os.path.join(HERE, "..", "include", "gelo.h")]
    jobs = []
    for src in sources:
        obj = os.path.join(OBJ, os.path.basename(src)[:-3] + ".o")
        if force or _stale(obj, [src] + headers):
            cmd = [_nvcc(), *NVCC_FLAGS, "-c", src, "-o", obj]
            if verbose:
                cmd.insert(1, "-Xptxas=-v")
            jobs.append(cmd)
    if jobs:
        with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(jobs))) as ex:
            for res in ex.map(lambda c: subprocess.run(c, capture_output=True, text=True), jobs):
                if verbose or res.returncode != 0:
                    sys.stderr.write(res.stdout + res.stderr)
                if res.returncode != 0:
                    raise RuntimeError("nvcc failed: " + " ".join(res.args))
    objs = [os.path.join(OBJ, os.path.basename(s)[:-3] + ".o") for s in sources]
    if force or jobs or _stale(LIB, objs):
        tmp = LIB + f".{os.getpid()}.tmp"
        subprocess.check_call([_nvcc(), "-shared", "-o", tmp, *objs, "-lcudart"])
        os.replace(tmp, LIB)
    _build_marshal(force)
    return LIB


def _torch_dir() -> str | None:
    spec = importlib.util.find_spec("torch")
    return os.path.dirname(spec.origin) if spec and spec.origin else None


def _build_marshal(force: bool) -> None:
    """``_marshal.so``: a Python module on torch's C++ tensors, linked against the ``libgelo.so`` beside it."""
    src = os.path.join(CSRC, "marshal.cpp")
    cuda, torch_dir, python = os.environ.get("CUDA_HOME", "/usr/local/cuda"), _torch_dir(), sysconfig.get_paths()["include"]
    missing = [] if torch_dir else ["torch"]
    for path in (os.path.join(python, "Python.h"), os.path.join(torch_dir or "", "include", "c10", "cuda", "CUDAStream.h"),
                 os.path.join(cuda, "include", "cuda_runtime_api.h")):
        if not os.path.exists(path):
            missing.append(path)
    if missing:
        if os.path.exists(MARSHAL):
            os.remove(MARSHAL)                                # it belongs to another installation
        sys.stderr.write(f"_marshal.so is not built, for want of {', '.join(missing)}\n")
        return
    made_for = f"{sysconfig.get_config_var('SOABI')} torch {importlib.metadata.version('torch')}"
    same = os.path.exists(MARSHAL_FOR) and open(MARSHAL_FOR).read() == made_for
    if not (force or not same or _stale(MARSHAL, [src, os.path.join(HERE, "..", "include", "gelo.h")])):
        return
    import torch
    torch_lib, torch_include = os.path.join(torch_dir, "lib"), os.path.join(torch_dir, "include")
    tmp = MARSHAL + f".{os.getpid()}.tmp"
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-isystem", torch_include, "-isystem", os.path.join(torch_include, "torch", "csrc", "api", "include"), "-isystem", os.path.join(cuda, "include"),
           "-isystem", python, src, "-o", tmp, f"-L{HERE}", "-l:libgelo.so", f"-L{torch_lib}", "-lc10", "-lc10_cuda",
           "-ltorch_cpu", "-ltorch_python", "-Wl,-rpath,$ORIGIN", f"-Wl,-rpath,{torch_lib}"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("g++ failed: " + " ".join(cmd))
    os.replace(tmp, MARSHAL)
    with open(MARSHAL_FOR, "w") as f:
        f.write(made_for)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
