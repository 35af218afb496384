"""Build libexactmoe.so (HIP for gfx950) in-tree with hipcc, and the compiled
half of the Python binding (_binding.so) with the host compiler.

    python -m paper_2608_15383_amd.build

Every call recompiles all sources; objects go to paper_2608_15383_amd/_build/
and the libraries to paper_2608_15383_amd/.
"""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libexactmoe.so")
BINDING = os.path.join(PKG, "_binding.so")
SOURCES = ["capi.hip", "quantize.hip", "route.hip", "gemv.hip", "gemm.hip", "decode.hip",
           "decoder.hip", "paged.hip", "logits.hip"]

CXX = os.environ.get("CXX", "g++")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # no packed-FP32 VALU instructions anywhere in the device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
    "-I", INCLUDE, "-I", CSRC,
]


def _run(cmd):
    proc = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in proc.stdout.splitlines() if "packed-fp32-ops" not in l
                    and "not a recognized feature" not in l)
    if proc.returncode != 0:
        raise RuntimeError(f"command failed ({proc.returncode}): {' '.join(cmd)}\n{out}")
    return out


def build_binding() -> str:
    """Compile csrc/binding.cpp against this interpreter and its PyTorch."""
    import torch
    root = os.path.dirname(torch.__file__)
    tmp = BINDING + ".tmp"
    _run([CXX, "-O2", "-std=c++17", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__",
          f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}", "-I", INCLUDE,
          "-I", os.path.join(root, "include"), "-I", sysconfig.get_paths()["include"],
          "-isystem", "/opt/rocm/include", os.path.join(CSRC, "binding.cpp"), "-o", tmp,
          "-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"])
    os.replace(tmp, BINDING)
    return BINDING


def build(verbose: bool = False, defines=(), lib: str = LIB, objdir: str = BUILD) -> str:
    """Compile every source and link `lib`; `defines` are extra -D macros
    (measurement variants such as EMOE_PHASE_TRACE go to their own objdir)."""
    os.makedirs(objdir, exist_ok=True)
    objs = []
    jobs = []
    for src in SOURCES:
        obj = os.path.join(objdir, src.replace(".hip", ".o"))
        objs.append(obj)
        jobs.append([HIPCC, *FLAGS, *[f"-D{m}" for m in defines], "-c", os.path.join(CSRC, src),
                     "-o", obj])
    with ThreadPoolExecutor(max_workers=min(len(jobs) + 1, os.cpu_count() or 4)) as ex:
        binding = ex.submit(build_binding) if lib == LIB else None
        for out in ex.map(_run, jobs):
            if verbose and out.strip():
                print(out)
        if binding:
            binding.result()
    tmp = lib + ".tmp"
    _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs,
          "-L/opt/rocm/lib", "-lrocblas", "-Wl,-rpath,/opt/rocm/lib"])
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
