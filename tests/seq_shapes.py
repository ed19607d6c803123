"""Routes of the sequence operators' calls: csrc/seq_shape.h through ctypes."""
import ctypes
import functools
import os
import subprocess
import tempfile
from types import SimpleNamespace

from paper_2101_09808_amd import build
from paper_2101_09808_amd.conv import CONV_DTYPE_BF16, CONV_DTYPE_F32

HERE = os.path.dirname(os.path.abspath(__file__))
SCAN = "rows waves steps segs seg_chunks fine fine_chunks chunks blks batch".split()
NORM = "flat nt cl tiles parts part wgs held".split()


@functools.lru_cache(None)
def _lib():
    with tempfile.TemporaryDirectory() as d:
        lib = os.path.join(d, "shapes.so")
        subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", build.INCLUDE, "-I", build.CSRC,
                        os.path.join(HERE, "seq_shape_harness.cpp"), "-o", lib], check=True)
        return ctypes.CDLL(lib)


def _call(f, names, *args):
    o = (ctypes.c_int64 * len(names))()
    getattr(_lib(), f)(*args, o)
    return SimpleNamespace(**dict(zip(names, o)))


def scan(N, D, L, S, G=1, bwd=False):
    return _call("t_scan", SCAN, N, D, L, S, G, int(bwd))


def norm(N, D, L, res_bf16):
    return _call("t_norm", NORM, N, D, L, CONV_DTYPE_BF16 if res_bf16 else CONV_DTYPE_F32)
