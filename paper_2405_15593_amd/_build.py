"""Builds libmicroadam.so (HIP for gfx950) in-tree with hipcc: every source
of csrc/ and csrc/ops/ is compiled to an object file in parallel, then linked.
Beside it _operators.so, the tensor side of some of its operators (csrc/torch/,
host code against torch's C++ headers)."""
from __future__ import annotations

import concurrent.futures as cf
import glob
import os
import subprocess
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OPS = os.path.join(CSRC, "ops")   # the operators beside the optimizer step
TORCH_SOURCE = os.path.join(CSRC, "torch", "operators.cpp")
INCLUDE = os.path.join(ROOT, "include")
LIBRARY = os.path.join(PKG, "libmicroadam.so")
OPERATORS = os.path.join(PKG, "_operators.so")
OBJDIR = os.path.join(PKG, "_build")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

COMPILE_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # one rounding per written operation: results that decide integers
    # (EF codes, Top-K) must not depend on FMA contraction
    "-ffp-contract=off",
    # no packed FP32 instructions in generated code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
    "-I", INCLUDE, "-I", CSRC,
]
# the optimizer step's device code: min/max without IEEE NaN quieting, so that
# they fuse with lane permutes (gradients are taken to be finite)
FINITE_FLAGS = ["-Xarch_device", "-fno-honor-nans", "-Xarch_device", "-mno-amdgpu-ieee"]
LINK_FLAGS = ["--offload-arch=gfx950", "-shared", "-fPIC", "-Wl,-rpath,/opt/rocm/lib"]


def _torch_flags() -> tuple[list[str], list[str]]:
    """(compiling, linking)"""
    import torch   # (not in every process that builds the library alone)
    at = os.path.dirname(torch.__file__)
    include = [os.path.join(at, "include"), os.path.join(at, "include", "torch", "csrc", "api", "include"),
               os.path.join(os.path.dirname(os.path.dirname(HIPCC)), "include"), sysconfig.get_paths()["include"]]
    return (["-O2", "-std=c++17", "-fPIC", "-Wall", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1",
             f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", INCLUDE,
             *(x for i in include for x in ("-isystem", i))],
            ["-shared", "-fPIC", "-L", PKG, "-L", os.path.join(at, "lib"), "-lmicroadam", "-lc10", "-lc10_hip",
             "-ltorch_cpu", "-ltorch_python", "-Wl,-rpath,$ORIGIN"])


def sources() -> list[str]:
    return sorted(f for d in (CSRC, OPS) for kind in ("*.hip", "*.cpp") for f in glob.glob(os.path.join(d, kind)))


def _compile(src: str) -> str:
    obj = os.path.join(OBJDIR, os.path.basename(src) + ".o")
    flags = COMPILE_FLAGS if os.path.dirname(src) == OPS else COMPILE_FLAGS + FINITE_FLAGS
    cmd = [HIPCC, *flags, "-x", "hip", "-c", src, "-o", obj + ".tmp"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed on {os.path.basename(src)} ({res.returncode}):\n{res.stderr[-6000:]}")
    os.replace(obj + ".tmp", obj)
    return obj


def _run(what: str, cmd: list[str], verbose: bool = False) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"{what} failed ({res.returncode}):\n{res.stderr[-6000:]}")


def _compile_torch() -> str:
    obj = os.path.join(OBJDIR, "torch_operators.cpp.o")
    _run("the compiler (operators.cpp)", [HIPCC, "-x", "c++", *_torch_flags()[0], "-c", TORCH_SOURCE, "-o", obj + ".tmp"])
    os.replace(obj + ".tmp", obj)
    return obj


def _link_torch(obj: str, verbose: bool = False) -> None:
    """(against the library as it was linked before)"""
    tmp = OPERATORS + ".tmp"
    _run("linking _operators.so", [HIPCC, obj, *_torch_flags()[1], "-o", tmp], verbose)
    os.replace(tmp, OPERATORS)


def build(verbose: bool = False, jobs: int | None = None) -> str:
    """Compiles every HIP/C++ source (always) and links both libraries."""
    os.makedirs(OBJDIR, exist_ok=True)
    srcs = sources()
    jobs = jobs or min(len(srcs), os.cpu_count() or 4, 16)
    with cf.ThreadPoolExecutor(jobs) as ex:
        torch_obj = ex.submit(_compile_torch)
        objs = list(ex.map(_compile, srcs))
    tmp = LIBRARY + ".tmp"
    _run("link", [HIPCC, *LINK_FLAGS, *objs, "-o", tmp], verbose)
    os.replace(tmp, LIBRARY)
    _link_torch(torch_obj.result(), verbose)
    return LIBRARY


if __name__ == "__main__":
    print(build(verbose=True))
