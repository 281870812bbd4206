"""Build libmoba.so (HIP, gfx950) in-tree with hipcc.

    python -m paper_2502_13189_amd.build

Every HIP source under csrc/ is compiled to an object in parallel, then linked
into paper_2502_13189_amd/libmoba.so; csrc/cache_binding.cpp becomes the Python module
paper_2502_13189_amd/_cache_binding.so, which calls it.  Packed fp32 instructions are disabled
for the device code (hipcc's host pass warns that it does not know the
feature; that warning is expected).
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libmoba.so")
MODULE = os.path.join(HERE, "_cache_binding.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"

DEVICE_FLAGS = ["-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
COMMON = ["-O3", "-std=c++17", "-fPIC", "--offload-arch=" + ARCH, "-I" + INCLUDE, "-I" + CSRC,
          "-Wall", "-Wno-unused-result"]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.basename(src) + ".o")
    cmd = [HIPCC, *COMMON, *DEVICE_FLAGS, "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    msgs = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                     if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s" % (src, msgs))
    if msgs.strip():
        sys.stderr.write(msgs + "\n")
    return obj


def _build_module() -> None:
    """The Python module (host code alone), against libmoba.so beside it and torch."""
    import sysconfig

    import torch

    at = os.path.dirname(torch.__file__)
    tmp = MODULE + ".tmp%d" % os.getpid()
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-D__HIP_PLATFORM_AMD__",
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
           "-I" + INCLUDE, "-isystem", "/opt/rocm/include",
           "-isystem", sysconfig.get_paths()["include"],
           "-isystem", os.path.join(at, "include"),
           "-isystem", os.path.join(at, "include", "torch", "csrc", "api", "include"),
           os.path.join(CSRC, "cache_binding.cpp"), "-o", tmp, "-L" + HERE, "-l:libmoba.so",
           "-Wl,-rpath,$ORIGIN", "-L" + os.path.join(at, "lib"), "-ltorch_python", "-ltorch",
           "-ltorch_cpu", "-lc10"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("g++ failed for cache_binding.cpp:\n" + r.stdout + r.stderr)
    if r.stderr.strip():
        sys.stderr.write(r.stderr)
    os.replace(tmp, MODULE)


def build(verbose: bool = False) -> str:
    """Compile every HIP source, link libmoba.so and build the module that calls it; returns
    the library's path."""
    os.makedirs(BUILD, exist_ok=True)
    srcs = sources()
    with cf.ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        objs = list(ex.map(_compile, srcs))
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [HIPCC, "--offload-arch=" + ARCH, "-shared", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stdout + r.stderr)
    os.replace(tmp, LIB)
    _build_module()
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
