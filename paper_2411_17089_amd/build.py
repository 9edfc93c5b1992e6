"""Builds libkvpr.so (HIP kernels + C ABI) for gfx950 with hipcc, and the binding's helper with the host compiler, in-tree."""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libkvpr.so")
OBJDIR = os.path.join(HERE, "_build")

HIP_SOURCES = ["context.hip", "store.hip", "profiler.hip", "kernels_abi.hip", "gemm_recompute.hip", "gemm_token.hip", "gemm_few.hip", "attention_decode.hip", "elementwise.hip", "store_int4.hip", "paged_abi.hip", "paged_plan.hip",
               "paged_cache.hip", "paged_attention.hip", "verify.hip"]
HOST_SOURCES = ["planner.cpp"]
ARGS_LIB = os.path.join(HERE, "_tensor_args.so")

COMMON = ["-O3", "-std=c++17", "-fPIC", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, "-Wall", "-Wno-unused-result"]
# packed-fp32 VALU forms are kept out of the generated code on purpose
HIP_FLAGS = ["--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _run(cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("build failed: %s\n%s\n%s" % (" ".join(cmd), r.stdout, r.stderr))
    return r


def _tensor_args_command():
    """_tensor_args.so: a Python module on torch's headers.  Its torch symbols are those of the torch that the binding has loaded."""
    torch_dir = importlib.util.find_spec("torch").submodule_search_locations[0]
    include = [sysconfig.get_paths()["include"], os.path.join(torch_dir, "include"), os.path.join(torch_dir, "include", "torch", "csrc", "api", "include")]
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", *("-I" + p for p in include), os.path.join(CSRC, "tensor_args.cpp"), "-o", ARGS_LIB,
            "-L" + os.path.join(torch_dir, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    os.makedirs(OBJDIR, exist_ok=True)
    jobs = []
    for src in HIP_SOURCES:
        obj = os.path.join(OBJDIR, src + ".o")
        jobs.append([hipcc, *COMMON, *HIP_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj])
    for src in HOST_SOURCES:
        obj = os.path.join(OBJDIR, src + ".o")
        jobs.append([hipcc, *COMMON, "-ffp-contract=off", "-x", "c++", "-c", os.path.join(CSRC, src), "-o", obj])
    objs = [j[-1] for j in jobs]
    jobs.append(_tensor_args_command())
    with ThreadPoolExecutor(max_workers=min(8, len(jobs))) as ex:
        list(ex.map(_run, jobs))
    _run([hipcc, "-shared", "-fPIC", "--offload-arch=gfx950", *objs, "-o", LIB])
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
