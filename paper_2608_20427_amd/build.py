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

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libbf1.so")
MARSHAL = os.path.join(HERE, "_marshal.so")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
ARCH = "gfx950"

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
    k_obj = os.path.join(BUILD, "bf1_kernels.o")
    b_obj = os.path.join(BUILD, "bf1_bwd.o")
    d_obj = os.path.join(BUILD, "bf1_decode.o")
    s_obj = os.path.join(BUILD, "bf1_stack.o")
    c_obj = os.path.join(BUILD, "bf1_cache.o")
    q_obj = os.path.join(BUILD, "bf1_decode_q8.o")
    a_obj = os.path.join(BUILD, "bf1_api.o")
    _run([hipcc, *HIP_FLAGS, *extra_hip_flags, "-c", os.path.join(CSRC, "bf1_kernels.hip"),
          "-o", k_obj], verbose)
    _run([hipcc, *HIP_FLAGS, *extra_hip_flags, "-c", os.path.join(CSRC, "bf1_bwd.hip"),
          "-o", b_obj], verbose)
    _run([hipcc, *HIP_FLAGS, *extra_hip_flags, "-c", os.path.join(CSRC, "bf1_decode.hip"),
          "-o", d_obj], verbose)
    _run([hipcc, *HIP_FLAGS, *extra_hip_flags, "-c", os.path.join(CSRC, "bf1_stack.hip"),
          "-o", s_obj], verbose)
    _run([hipcc, *HIP_FLAGS, *extra_hip_flags, "-c", os.path.join(CSRC, "bf1_cache.hip"),
          "-o", c_obj], verbose)
    _run([hipcc, *HIP_FLAGS, *extra_hip_flags, "-c", os.path.join(CSRC, "bf1_decode_q8.hip"),
          "-o", q_obj], verbose)
    _run([gxx, *HOST_FLAGS, "-c", os.path.join(CSRC, "bf1_api.cpp"), "-o", a_obj], verbose)
    tmp = LIB + ".tmp"
    _run([hipcc, f"--offload-arch={ARCH}", "-shared", "-fPIC", k_obj, b_obj, d_obj, s_obj, c_obj, q_obj, a_obj,
          "-o", tmp,
          f"-L{ROCM}/lib", "-lamdhip64", f"-Wl,-rpath,{ROCM}/lib"], verbose)
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
