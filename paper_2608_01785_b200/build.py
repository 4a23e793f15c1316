"""Builds the C-ABI shared library (CUDA kernels for sm_100a + host code) with nvcc, and the Python binding of its device-resident operators with
the host compiler, both in-tree."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libhorizonserve.so")
BINDING = os.path.join(_HERE, "_device_binding.so")
SOURCES = ["api.cu", "gemm.cu", "gemm_skinny.cu", "small_step.cu", "metadata.cu", "attention.cu", "attention_prefill.cu", "norm.cu", "noalloc.cu", "diag.cu", "head.cu", "step_tables.cu", "rope_cache.cu", "paged_decode.cu",
           "paged_chunk.cu", "token_logprobs.cu", "beam_select.cu", "shared_pages.cu", "shared_attention.cu", "device_api.cu", "plan.cc", "control.cc"]
HEADERS = ["hs_internal.h", "kernels.h", "ptx.cuh", "attention_decode.cuh", "weight_stream.cuh", "device_ops.h", "paged_scores.cuh", "paged_tiles.cuh", "block_scan.cuh",
           os.path.join("..", "..", "include", "horizonserve.h"),
           os.path.join("..", "..", "include", "horizonserve_ops.h"),
           os.path.join("..", "..", "include", "horizonserve_control.h"),
           os.path.join("..", "..", "include", "horizonserve_head.h"),
           os.path.join("..", "..", "include", "horizonserve_device.h"),
           os.path.join("..", "..", "include", "horizonserve_beams.h")]
NVCC_FLAGS = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden", "--expt-relaxed-constexpr"]


def _older(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in [*deps, os.path.abspath(__file__)])


def _stale() -> bool:
    return _older(LIB, [os.path.join(CSRC, f) for f in SOURCES + HEADERS])


def _binding_stale() -> bool:
    return _older(BINDING, [os.path.join(CSRC, "device_binding.cpp"), *(os.path.join(CSRC, "..", "..", "include", f"horizonserve{n}.h") for n in ("", "_device", "_beams"))])


def _start_binding():
    """Starts the compiler of _device_binding.so, against the torch that is installed.  (The name changes in one step, so that a process that has
    the old file mapped keeps it.)"""
    import torch
    root = os.path.dirname(torch.__file__)
    include = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"],
               os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *[w for i in include for w in ("-isystem", i)], os.path.join(CSRC, "device_binding.cpp"), "-o", BINDING + ".tmp", "-L" + os.path.join(root, "lib"),
           *("-l" + n for n in ("c10", "c10_cuda", "torch_cpu", "torch_cuda", "torch", "torch_python"))]
    return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def _end_binding(p) -> None:
    out, _ = p.communicate()
    if p.returncode != 0:
        print(f"--- device_binding.cpp\n{out}", file=sys.stderr)
        raise RuntimeError("the host compiler failed")
    os.replace(BINDING + ".tmp", BINDING)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compiles every source for sm_100a and links libhorizonserve.so next to this file; _device_binding.so beside it."""
    binding = _start_binding() if force or _binding_stale() else None
    if force or _stale():
        _build_library(verbose)
    if binding is not None:
        _end_binding(binding)
    return LIB


def _build_library(verbose: bool) -> None:
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    objs = []
    procs = []
    obj_dir = os.path.join(_HERE, "build")
    os.makedirs(obj_dir, exist_ok=True)
    for src in SOURCES:
        obj = os.path.join(obj_dir, src + ".o")
        cmd = [nvcc, *NVCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas")
            cmd.insert(2, "-v")
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        if out.strip() and (verbose or p.returncode != 0):
            print(f"--- {src}\n{out}", file=sys.stderr)
        failed |= p.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed")
    subprocess.run([nvcc, "-shared", "-o", LIB, *objs, "-cudart", "static"], check=True)


if __name__ == "__main__":
    build(force=True, verbose="-v" in sys.argv)
    print(LIB)
