"""Builds the CUDA library in-tree: ``libpatch_b200.so`` next to this file (sm_100a only)."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libpatch_b200.so")
LIB_FI = os.path.join(HERE, "libpatch_b200_fi.so")
SOURCES = ["pack.cu", "masks.cu", "gemv.cu", "gemm_decode_sm100.cu", "gemm_decode_cluster_sm100.cu", "gemm_prefill_sm100.cu", "gemm_prefill2_sm100.cu", "gemm_prefill_pair_sm100.cu", "gemm_prefill_pair_mixed_sm100.cu", "gemm_decode_q4_sm100.cu",
           "qk_rope.cu", "attention.cu", "attention_decode_sm100.cu", "attention_block_sm100.cu", "api.cu"]


MARSHAL = os.path.join(HERE, "_marshal.so")
MARSHAL_SRC = os.path.join(CSRC, "marshal.cpp")


def _stale(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    deps = [MARSHAL_SRC] if lib == MARSHAL else [os.path.join(CSRC, f) for f in os.listdir(CSRC)
                                                 if os.path.isfile(os.path.join(CSRC, f)) and not f.endswith(".cpp")]
    deps.append(os.path.join(os.path.dirname(HERE), "include", "patch.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def build_marshal(force: bool = False) -> str:
    """The CPython module that takes torch tensors apart for the calls of a few microseconds (g++, Python's and torch's headers).  It holds
    the version of the torch it was built against and is built again for another one."""
    import sysconfig
    import torch
    mark = f"for torch {torch.__version__}"
    if not (force or _stale(MARSHAL)):
        with open(MARSHAL, "rb") as f:
            if mark.encode() + b"\0" in f.read():
                return MARSHAL
    root = os.path.dirname(torch.__file__)
    inc, lib = os.path.join(root, "include"), os.path.join(root, "lib")
    abi = int(torch._C._GLIBCXX_USE_CXX11_ABI)
    subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={abi}",
                    f'-DPATCH_BUILT="{mark}"', f"-I{inc}",
                    "-I" + os.path.join(inc, "torch", "csrc", "api", "include"), "-I" + sysconfig.get_paths()["include"], "-o", MARSHAL,
                    MARSHAL_SRC, f"-L{lib}", "-ltorch_python", "-ltorch_cpu", "-lc10", f"-Wl,-rpath,{lib}"], check=True)
    return MARSHAL


def build(force: bool = False, verbose: bool = False, fault_injection: bool = False) -> str:
    """The library; with ``fault_injection`` the test build ``libpatch_b200_fi.so`` (same sources with
    -DPATCH_FAULT_INJECTION: device-side waits give up after 300 us, and decode and attention kernels can be told,
    through their status word, to announce bytes that never arrive -- how the tests make a bounded wait run out).  The library
    needs nvcc alone.  The module for torch's tensors is built along with it where torch and its headers are; where it cannot be, that is
    said on stderr and the binding's calls that use it raise."""
    lib = LIB_FI if fault_injection else LIB
    if force or _stale(lib):
        _compile(lib, verbose, fault_injection)
    try:
        build_marshal(force and not fault_injection)
    except (ImportError, OSError, subprocess.CalledProcessError) as e:
        print(f"{MARSHAL} was not built ({e}): the C library is complete, the binding's calls between the linear layers need it", file=sys.stderr)
    return lib


def _compile(lib: str, verbose: bool, fault_injection: bool) -> None:
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-Xcompiler", "-fPIC", "-shared", "-cudart", "static", "-o", lib]
    if fault_injection:
        cmd += ["-DPATCH_FAULT_INJECTION"]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    subprocess.run(cmd, check=True)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, fault_injection="--fault-injection" in sys.argv))
