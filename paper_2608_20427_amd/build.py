"""Build libbf1.so in-tree for gfx950.

    python -m paper_2608_20427_amd.build          # or __graft_entry__.build()

The device code is compiled by hipcc for gfx950 only; the C-ABI shim is plain
host C++ (g++ against the HIP runtime headers), and so is _marshal.so, the native
marshalling of the cache's operators (against torch's headers; torch itself is not
imported).  Packed FP32 VALU forms are disabled in device code on purpose.
"""

import importlib.util

import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libbf1.so")
MARSHAL = os.path.join(HERE, "_marshal.so")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
ARCH = "gfx950"
HIP_SOURCES = ("bf1_tree", "bf1_decode", "bf1_decode_q8", "bf1_kernels", "bf1_bwd", "bf1_norm_rope", "bf1_cache",
               "bf1_stack", "bf1_pages")

HIP_FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]
HOST_FLAGS = ["-O2", "-std=c++17", "-fPIC", "-Wall", "-Wextra",
              f"-I{ROCM}/include", "-D__HIP_PLATFORM_AMD__"]


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in r.stdout.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"build step failed ({r.returncode}): {' '.join(cmd)}\n{out}")
    if verbose and out.strip():
        print(out, flush=True)


def build(verbose=False, extra_hip_flags=()):
    hipcc = shutil.which("hipcc") or os.path.join(ROCM, "bin", "hipcc")
    gxx = shutil.which("g++") or "g++"
    os.makedirs(BUILD, exist_ok=True)
    objs, steps = [], []
    for name in HIP_SOURCES:
        objs.append(os.path.join(BUILD, name + ".o"))
        steps.append([hipcc, *HIP_FLAGS, *extra_hip_flags, "-c", os.path.join(CSRC, name + ".hip"), "-o", objs[-1]])
    objs.append(os.path.join(BUILD, "bf1_api.o"))
    steps.append([gxx, *HOST_FLAGS, "-c", os.path.join(CSRC, "bf1_api.cpp"), "-o", objs[-1]])
    with ThreadPoolExecutor(4) as pool:
        list(pool.map(lambda cmd: _run(cmd, verbose), steps))
    tmp = LIB + ".tmp"
    _run([hipcc, f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp, f"-L{ROCM}/lib", "-lamdhip64",
          f"-Wl,-rpath,{ROCM}/lib"], verbose)
    os.replace(tmp, LIB)
    torch = importlib.util.find_spec("torch").submodule_search_locations[0]
    inc, lib = os.path.join(torch, "include"), os.path.join(torch, "lib")
    tmp = MARSHAL + ".tmp"
    _run([gxx, "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-D__HIP_PLATFORM_AMD__", "-DUSE_ROCM",
          "-D_GLIBCXX_USE_CXX11_ABI=1", "-isystem", inc, "-isystem", os.path.join(inc, "torch", "csrc", "api", "include"),
          "-isystem", sysconfig.get_paths()["include"], "-isystem", f"{ROCM}/include",
          os.path.join(CSRC, "bf1_torch.cpp"), "-o", tmp, f"-L{lib}", "-lc10", "-lc10_hip", "-ltorch_cpu",
          "-ltorch_python", f"-L{HERE}", "-l:libbf1.so", "-Wl,-rpath,$ORIGIN"], verbose)
    os.replace(tmp, MARSHAL)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
