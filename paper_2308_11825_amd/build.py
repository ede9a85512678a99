"""Builds libagcn.so (HIP, gfx950) in-tree with hipcc, and _binding.so (the compiled part of the
Python binding) with g++.

Usage: python -m paper_2308_11825_amd.build
"""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
LIB_PATH = os.path.join(PKG, "libagcn.so")
BINDING_PATH = os.path.join(PKG, "_binding.so")
CSRC = os.path.join(PKG, "csrc")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

# Packed fp32 instructions are kept out of every kernel: the compiler may not
# form them (the target feature is switched off) and none are written by hand.
HIP_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"),
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def _hipcc(args, out_path, verbose):
    tmp = out_path + ".tmp"
    cmd = [HIPCC, *HIP_FLAGS, *args, "-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    out = res.stdout + res.stderr
    # The host pass does not know the packed-fp32 target feature and says so.
    noise = "is not a recognized feature for this target"
    lines = [l for l in out.splitlines() if noise not in l and "(ignoring feature)" not in l]
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + "\n".join(lines))
    if verbose and lines:
        print("\n".join(lines), flush=True)
    os.replace(tmp, out_path)


def build(verbose: bool = False) -> str:
    """Compile every HIP source into libagcn.so, several at a time, and the binding. Always
    recompiles."""
    with tempfile.TemporaryDirectory() as to:
        jobs = [(src, os.path.join(to, os.path.basename(src) + ".o")) for src in sources()]
        jobs.sort(key=lambda job: -os.path.getsize(job[0]))
        with ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
            binding = pool.submit(build_binding, verbose)
            list(pool.map(lambda job: _hipcc(["-c", job[0]], job[1], verbose), jobs))
            binding.result()
        _hipcc(["-shared", *[o for _, o in jobs]], LIB_PATH, verbose)
    return LIB_PATH


def build_binding(verbose: bool = False) -> str | None:
    """Compile _binding.so against the installed PyTorch; without one built for ROCm there is
    none to build, and libagcn.so serves C callers. It takes the library's functions by their
    addresses, so the two can be built in any order."""
    try:
        import torch
    except ImportError:
        torch = None
    if torch is None or torch.version.hip is None:
        print("no PyTorch for ROCm: libagcn.so without its compiled Python binding", flush=True)
        return None
    top = os.path.dirname(torch.__file__)
    lib = os.path.join(top, "lib")
    tmp = BINDING_PATH + ".tmp"
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-D__HIP_PLATFORM_AMD__=1",
           "-DUSE_ROCM=1", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-isystem", os.path.join(top, "include"), "-isystem", "/opt/rocm/include",
           "-isystem", sysconfig.get_paths()["include"], os.path.join(CSRC, "agcn_binding.cpp"), "-o", tmp,
           "-L", lib, "-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch_python", "-Wl,-rpath," + lib]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("g++ failed:\n" + res.stdout + res.stderr)
    if verbose and res.stderr:
        print(res.stderr, flush=True)
    os.replace(tmp, BINDING_PATH)
    return BINDING_PATH


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
