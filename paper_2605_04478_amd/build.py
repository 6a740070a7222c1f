"""Builds libccld.so (the HIP library, gfx950) and _step.so (the calls of a training step's operators from Python) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libccld.so")
SOURCES = ("radix_sort.hip", "window.hip", "segments.hip", "groups.hip", "grid.hip", "merge.hip", "chains.hip", "hang.hip", "api.hip",
           "experts.hip", "join.hip", "vocab_loss.hip", "norms.hip", "routing.hip", "exchange.hip", "adamw.hip", "logprobs.hip")
STEP_SOURCE, STEP = os.path.join(CSRC, "step_calls.cpp"), os.path.join(HERE, "_step.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ROCM_INCLUDE = os.path.join(os.path.dirname(os.path.dirname(HIPCC)), "include")
FLAGS = ["-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-Wall", "-Wno-unused-function",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _step_commands():
    """Compiles and links _step.so: host code against torch's headers and libraries, which are loaded with torch."""
    import torch
    at = os.path.dirname(torch.__file__)
    obj = STEP_SOURCE.replace(".cpp", ".o")
    yield [HIPCC, "-x", "c++", "-O2", "-std=c++17", "-fPIC", "-Wall", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"),
           "-isystem", ROCM_INCLUDE, "-isystem", os.path.join(at, "include"), "-isystem", os.path.join(at, "include", "torch", "csrc", "api", "include"),
           "-isystem", sysconfig.get_paths()["include"], "-c", STEP_SOURCE, "-o", obj]
    yield [HIPCC, "-shared", "-fPIC", "-o", STEP, obj, LIB, "-Wl,-rpath,$ORIGIN", "-L", os.path.join(at, "lib"),
           "-ltorch_python", "-ltorch_cpu", "-ltorch_hip", "-lc10", "-lc10_hip"]


def build_lib(verbose: bool = False) -> str:
    """Compile every translation unit for gfx950 and link the shared libraries."""
    objs = []

    def cc(src):
        obj = os.path.join(CSRC, src.replace(".hip", ".o"))
        cmd = [HIPCC] + FLAGS + ["-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.check_call(cmd)
        return obj

    srcs = [s for s in SOURCES if os.path.exists(os.path.join(CSRC, s))]
    compile_step, link_step = _step_commands()
    with ThreadPoolExecutor(max_workers=4) as ex:
        step = ex.submit(subprocess.check_call, compile_step)
        objs = list(ex.map(cc, srcs))
        step.result()
    subprocess.check_call([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-Wl,-soname,libccld.so", "-o", LIB] + objs)
    subprocess.check_call(link_step)
    return LIB


if __name__ == "__main__":
    print(build_lib(verbose="-v" in sys.argv))
