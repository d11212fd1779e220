"""Builds the CUDA library in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmx_b200.so")
PY_CALL = os.path.join(HERE, "_py_call.so")  # the Python side's marshalling module (csrc/py_call.cpp)
BUILD = os.path.join(HERE, "build")
STAMP = os.path.join(BUILD, "py_call.stamp")  # the interpreter and torch that module was compiled for
SOURCES = ["mx_api.cu", "mx_quantize.cu", "mx_quantize_dual.cu", "mx_quantize_tile.cu", "mx_dequantize.cu",
           "mx_gemm.cu", "mx_im2col.cu", "mx_rmsnorm.cu", "mx_route.cu", "mx_moe.cu", "mx_gemm_grouped.cu",
           "mx_kv.cu", "mx_kv_attention.cu", "mx_kv_attention_e4m3.cu", "mx_kv_attention_e5m2.cu",
           "mx_kv_attention_e2m1.cu", "mx_kv_attention_int8.cu"]
NVCC_FLAGS = ["-std=c++17", "-O3", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _newest_source() -> float:
    files = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "mx.h")]
    return max(os.path.getmtime(f) for f in files)


def py_call_for() -> str:
    """What the marshalling module depends on beside its sources: the C++ interfaces of this interpreter and torch.
    Empty without torch."""
    try:
        import torch
    except ImportError:
        return ""
    return f"python {sys.version_info[0]}.{sys.version_info[1]}, torch {torch.__version__}"


def _stale_py_call() -> bool:
    """The marshalling module is missing, older than a source or compiled for another interpreter or torch."""
    want = py_call_for()
    if not want:
        return False  # nobody here can call it
    if not os.path.exists(PY_CALL) or not os.path.exists(STAMP):
        return True
    if os.path.getmtime(PY_CALL) < max(os.path.getmtime(f) for f in (os.path.join(CSRC, "py_call.cpp"), os.path.join(ROOT, "include", "mx.h"))):
        return True
    with open(STAMP) as f:
        return f.read() != want


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(BUILD, src.replace(".cu", ".o"))
    deps = [os.path.join(CSRC, src), os.path.join(ROOT, "include", "mx.h")] + \
           [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    if os.path.exists(obj) and os.path.getmtime(obj) >= max(os.path.getmtime(d) for d in deps):
        return obj
    cmd = ["nvcc", *NVCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
    subprocess.check_call(cmd)
    return obj


def _build_py_call() -> None:
    """Compile the marshalling module with g++ against torch's headers.  Its torch libraries are those of
    the process that imports it; the C library is found next to it."""
    import sysconfig

    import torch
    from torch.utils.cpp_extension import include_paths
    lib_dir = os.path.join(os.path.dirname(torch.__file__), "lib")
    cuda_inc = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(shutil.which("nvcc")))), "include")
    inc = [*include_paths(), sysconfig.get_paths()["include"], cuda_inc, os.path.join(ROOT, "include")]
    tmp = PY_CALL + f".tmp{os.getpid()}"
    subprocess.check_call(["g++", "-std=c++20", "-O2", "-fPIC", "-shared", "-fvisibility=hidden",
                           f'-DMX_PY_CALL_FOR="{py_call_for()}"', os.path.join(CSRC, "py_call.cpp"), "-o", tmp,
                           *[f for i in inc for f in ("-isystem", i)], "-L", lib_dir, "-L", HERE, "-Wl,-rpath,$ORIGIN",
                           "-lmx_b200", "-ltorch_python", "-ltorch", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda"])
    os.replace(tmp, PY_CALL)
    with open(STAMP, "w") as f:
        f.write(py_call_for())


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every kernel file and link ``libmx_b200.so`` next to this module; where there is a torch, compile the
    marshalling module against it (again when torch or the interpreter has changed)."""
    have_lib = not force and os.path.exists(LIB)
    if have_lib and shutil.which("nvcc") is None:
        return LIB  # no compiler on this machine: use what was shipped
    os.makedirs(BUILD, exist_ok=True)
    if not have_lib or os.path.getmtime(LIB) < _newest_source():
        if force:
            for f in os.listdir(BUILD):
                if f.endswith(".o"):
                    os.remove(os.path.join(BUILD, f))
        with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
            objs = list(ex.map(lambda s: _compile(s, verbose), SOURCES))
        tmp = LIB + f".tmp{os.getpid()}"
        subprocess.check_call(["nvcc", "-shared", "-cudart", "static", "-gencode",
                               "arch=compute_100a,code=sm_100a", "-o", tmp, *objs])
        os.replace(tmp, LIB)
    if (force and py_call_for()) or _stale_py_call():
        _build_py_call()
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
