"""Compile the HIP sources into paper_2509_15038_amd/libcurdkv.so for gfx950, and the CPython module
_call and _attend beside it (argument marshalling, no device code; their file names end as this interpreter's modules do).

    python -m paper_2509_15038_amd.build

hipcc cross-compiles without a GPU.  Nothing is built lazily at import time:
tests, the smoke check and the benchmark load the library this step left here.
"""

from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libcurdkv.so")
CALL = os.path.join(HERE, "_call" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
ATTEND_CALL = os.path.join(HERE, "_attend" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
SOURCES = ["curdkv_api.hip", "scores_kernels.hip", "select_kernels.hip", "split_select.hip", "compact_kernels.hip", "fused_kernel.hip", "adaptive_kernels.hip",
           "sketch_host.cpp"]
ATTENTION = ["rotate_kernel.hip", "mx_kernels.hip", "attend_split.hip", "attend_prompt.hip", "attend_prompt_f32.hip", "attend_api.hip",
             "weights_kernels.hip", "evict_kernels.hip", "attend_shared.hip", "cache_api.hip"]


def _build_call_module(hipcc: str, verbose: bool, source=("csrc", "call_module.cpp"), to=None) -> None:
    """A CPython module.  Where there is no Python.h or no C++ compiler the binding does without it."""
    to = CALL if to is None else to
    headers = sysconfig.get_paths()["include"]
    compilers = [os.environ.get("CXX"), "g++", "clang++", os.path.join(os.path.dirname(hipcc), "amdclang++")]
    cxx = next((path for path in map(shutil.which, filter(None, compilers)) if path), None)
    if not cxx or not os.path.exists(os.path.join(headers, "Python.h")):
        if os.path.exists(to):                      # (of an older source)
            os.remove(to)
        print("no Python.h or no C++ compiler: the binding marshals its arguments through ctypes (1 us a call slower)", flush=True)
        return
    cmd = [cxx, "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-I", headers, "-I", os.path.join(ROOT, "include"),
           os.path.join(HERE, *source), "-o", to]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)


def build(verbose: bool = True) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    cmd = [hipcc, "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-shared",
           "-fno-gpu-rdc", "-Wall", "-Wno-unused-function",
           # packed fp32 VALU forms are switched off for all device code
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-I", os.path.join(ROOT, "include"), "-I", os.path.join(HERE, "csrc")]
    cmd += ["-x", "hip"] + [os.path.join(HERE, "csrc", s) for s in SOURCES] + [os.path.join(HERE, "attention", s) for s in ATTENTION]
    cmd += ["-o", LIB]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    _build_call_module(hipcc, verbose)
    _build_call_module(hipcc, verbose, ("attention", "attend_call.cpp"), ATTEND_CALL)
    return LIB


if __name__ == "__main__":
    build()
    print("built", LIB)
    sys.exit(0)
