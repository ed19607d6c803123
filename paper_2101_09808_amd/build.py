"""Build the HIP library ``libconvfwd.so`` in-tree for gfx950 with hipcc, and
the Python module ``_seq.so`` (the sequence operators' calls) on it with g++ and
torch's and Python's headers.

    python -m paper_2101_09808_amd.build
    python -m paper_2101_09808_amd.build --library    # libconvfwd.so alone
"""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libconvfwd.so")
SEQ = os.path.join(PKG, "_seq.so")
INCLUDE = os.path.join(os.path.dirname(PKG), "include")

SOURCES = ("conv_kernels.hip", "split_kernels.hip", "seq_scan.hip", "seq_norm.hip", "seq_conv.hip",
           "conv_api.cpp", "select.cpp", "split_route.cpp", "workspace.cpp", "seq_api.cpp")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"
# host sources call the HIP runtime (hipcc adds its headers to device sources only)
HOST_FLAGS = ["-D__HIP_PLATFORM_AMD__", "-I", os.path.join(os.path.dirname(os.path.dirname(HIPCC)), "include")]
# Packed fp32 instructions are disabled for all device code.
DEVICE_FLAGS = ["-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
COMMON = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}", "-I", INCLUDE, "-I", CSRC,
          "-Wall", "-Wno-unused-function", "-Wno-pass-failed"]


def _compile(src):
    out = os.path.join(OBJ, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *COMMON, *DEVICE_FLAGS, "-c", os.path.join(CSRC, src), "-o", out]
    if src.endswith(".cpp"):
        cmd = [HIPCC, *COMMON, *HOST_FLAGS, "-x", "c++", "-c", os.path.join(CSRC, src), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True)
    msgs = [ln for ln in (r.stdout + r.stderr).splitlines() if "packed-fp32-ops" not in ln]
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n" + "\n".join(msgs))
    return out, msgs


def _build_python(verbose):
    """The module _seq (host code on torch's and Python's headers): its calls go to LIB."""
    import sysconfig

    import torch

    torch_dir = os.path.dirname(torch.__file__)
    tmp = SEQ + ".tmp%d" % os.getpid()
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-shared", "-Wall", "-DUSE_ROCM",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *HOST_FLAGS, "-I", INCLUDE,
           "-isystem", os.path.join(torch_dir, "include"),
           "-isystem", os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"),
           "-isystem", sysconfig.get_paths()["include"], os.path.join(CSRC, "seq_python.cpp"), "-o", tmp,
           "-L", PKG, "-lconvfwd", "-L", os.path.join(torch_dir, "lib"), "-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch_hip",
           "-ltorch_python", "-Wl,-rpath,$ORIGIN"]
    try:
        r = subprocess.run(cmd, capture_output=True, text=True)
    except OSError as e:
        raise RuntimeError(f"{LIB} is built, the Python module is not: {e}") from e
    if r.returncode != 0:
        raise RuntimeError(f"{LIB} is built, the Python module is not: {' '.join(cmd)}\n{r.stdout}{r.stderr}")
    if verbose and (r.stdout or r.stderr):
        print(r.stdout + r.stderr)
    os.replace(tmp, SEQ)


def build_library(verbose=False):
    """libconvfwd.so, which needs hipcc and nothing else."""
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        results = list(ex.map(_compile, SOURCES))
    objs = [o for o, _ in results]
    if verbose:
        for _, msgs in results:
            for m in msgs:
                print(m)
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stdout}{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


def build(verbose=False):
    build_library(verbose)
    _build_python(verbose)
    return LIB


if __name__ == "__main__":
    print((build_library if "--library" in sys.argv else build)(verbose="-v" in sys.argv))
