"""Build libsaki.so in-tree for gfx950.

The host calibration (C++17, float64) is compiled with g++ and the HIP
kernels with hipcc; hipcc links both into paper_2608_03228_amd/libsaki.so.
The Python binding's argument module (_saki_args) links to it.
Run ``python -m paper_2608_03228_amd.build`` (or call ``build()``).
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libsaki.so")
ARGS = os.path.join(PKG, "_saki_args" + sysconfig.get_config_var("EXT_SUFFIX"))
BUILD_DIR = os.path.join(PKG, "_build")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"
KERNELS = ("saki_kernels", "saki_serve", "saki_prompt",  # the index, and serving around it
           "saki_cache4", "saki_chunk4")  # a cache held in 4 bits
# Packed FP32 instructions are disabled for all device code.
NO_PACKED_FP32 = ["-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
# MFMA results are written to the architectural VGPRs rather than the
# accumulation registers, which saves a copy of every result the kernels
# inspect (the selection passes read each score).
MFMA_VGPR = ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]


def _run(cmd, verbose):
    if verbose:
        print("+", " ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)


def build(verbose: bool = True) -> str:
    """Compile every source and link libsaki.so; returns its path."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    host_o = os.path.join(BUILD_DIR, "saki_host.o")
    dev_o = [os.path.join(BUILD_DIR, name + ".o") for name in KERNELS]
    _run(["g++", "-O3", "-std=c++17", "-fPIC", "-march=x86-64-v3", "-pthread",
          "-Wall", "-Wextra", "-I", INCLUDE, "-I", CSRC, "-c",
          os.path.join(CSRC, "saki_host.cpp"), "-o", host_o], verbose)
    for name, obj in zip(KERNELS, dev_o):
        _run([HIPCC, "-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}", *NO_PACKED_FP32,
              *MFMA_VGPR, "-I", INCLUDE, "-I", CSRC, "-c", os.path.join(CSRC, name + ".hip"),
              "-o", obj], verbose)
    tmp = LIB + ".tmp"
    _run([HIPCC, "-shared", "-fPIC", f"--offload-arch={ARCH}", "-pthread", host_o, *dev_o,
          "-o", tmp], verbose)
    os.replace(tmp, LIB)
    build_args(verbose)
    return LIB


def build_args(verbose: bool = True) -> str:
    """Compile the binding's argument module against libsaki.so and torch."""
    import torch
    from torch.utils.cpp_extension import include_paths, library_paths
    tmp = ARGS + ".tmp"
    inc = [f for p in include_paths() for f in ("-isystem", p)]
    libs = [f for p in library_paths() for f in ("-L", p)]
    _run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-Wall", "-Wextra",
          f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", INCLUDE, *inc,
          "-I", sysconfig.get_paths()["include"], os.path.join(CSRC, "saki_args.cpp"),
          "-L", PKG, "-l:libsaki.so", "-Wl,-rpath,$ORIGIN", *libs, "-ltorch_python", "-ltorch_cpu",
          "-lc10",
          "-o", tmp], verbose)
    os.replace(tmp, ARGS)
    return ARGS


def clean():
    shutil.rmtree(BUILD_DIR, ignore_errors=True)
    for path in (LIB, ARGS):
        if os.path.exists(path):
            os.remove(path)


if __name__ == "__main__":
    build(verbose="-q" not in sys.argv)
