"""Builds libcornenc.so (HIP kernels + C ABI) for gfx950 with hipcc, and _calls.so (tensors in, C arguments out) beside it."""
from __future__ import annotations

import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcornenc.so")
CALLS = os.path.join(HERE, "_calls.so")
SOURCES = ["api.cpp", "plan.cpp", "channel.cpp", "xchannel.cpp", "gemm.hip", "attention.hip", "elementwise.hip", "probe.hip",
           "cache_api.cpp", "cache.hip", "cache_attention.hip", "block_api.cpp", "block.hip", "packed.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-x", "hip",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wall", "-Wno-unused-function"]


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(CSRC, os.path.splitext(src)[0] + ".o")
    cmd = ["hipcc", *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{err}")
    if verbose and err.strip():
        print(err)
    return obj


def build_calls() -> str:
    """The extension module of binding.py's hot calls: host code only, linked to the library beside it and to torch (whose C++ headers,
    like Python's and g++, nothing else here needs).  Without it the library's other calls run, and these say what is missing."""
    import sysconfig
    import torch
    if os.path.exists(CALLS):                  # (one that does not compile any more is not to answer for the library of now)
        os.remove(CALLS)
    root = os.path.dirname(torch.__file__)
    libs = os.path.join(root, "lib")
    include = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"), "/opt/rocm/include",
               sysconfig.get_paths()["include"]]
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *[x for i in include for x in ("-isystem", i)],
           os.path.join(CSRC, "calls.cpp"), "-o", CALLS, "-L" + libs, "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_hip", "-L" + HERE,
           "-l:libcornenc.so", "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("g++ failed on calls.cpp:\n" + r.stderr)
    return CALLS


def build_library(verbose: bool = False) -> str:
    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose), SOURCES))
    r = subprocess.run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
    print(build_calls())
