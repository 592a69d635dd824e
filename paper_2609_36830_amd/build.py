"""Build libpace.so (HIP for gfx950) in-tree with hipcc, and the extension _lists.so, which reads lists of tensors, with g++.

Every translation unit is compiled as HIP for gfx950 only, with IEEE binary64
arithmetic kept unfused (-ffp-contract=off) so scores are reproducible, and
with packed FP32 instructions disabled.
"""
from __future__ import annotations

import os
import subprocess
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libpace.so")
LISTS = os.path.join(HERE, "_lists.so")
SOURCES = ["score.hip", "score_traj.hip", "select.hip", "select_wide.hip", "compact.hip", "filter_step.hip", "group.hip", "stream.hip", "prefix.hip", "diag.hip", "logprob.hip", "policy_loss.hip", "matmul_i8.hip", "ortho.hip", "layer_norm.hip", "adamw.hip", "validate.hip", "noalloc.hip", "pace_abi.cpp"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["-x", "hip", "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         "-ffp-contract=off", "-fno-fast-math", "-Wall", "-Wno-pass-failed",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    subprocess.check_call([HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj],
                          stderr=subprocess.STDOUT)
    return obj


def _compile_lists() -> None:
    """The extension against torch's headers and libraries; those are loaded already wherever it is."""
    import torch
    home = os.path.dirname(torch.__file__)
    tmp = LISTS + ".tmp%d" % os.getpid()
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-Wall",
                           "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
                           "-isystem", os.path.join(home, "include"), "-isystem", sysconfig.get_paths()["include"],
                           os.path.join(CSRC, "tensor_lists.cpp"), "-o", tmp,
                           "-L" + os.path.join(home, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"])
    os.replace(tmp, LISTS)


def build() -> str:
    """Compile every source and link libpace.so and _lists.so; returns the former's path."""
    os.makedirs(BUILD, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(len(SOURCES) + 1, os.cpu_count() or 1)) as ex:
        lists = ex.submit(_compile_lists)
        objs = list(ex.map(_compile, SOURCES))
        lists.result()
    tmp = LIB + ".tmp%d" % os.getpid()
    subprocess.check_call([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build())
