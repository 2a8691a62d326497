"""The library's own choice of a kernel by a call's sizes
(paper_2606_24031_amd/csrc/choice.h), compiled for the host: tests that mean to
reach a kernel ask it."""
import collections
import ctypes
import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
Q8_WAYS = ("few 1x1", "few 1x2", "few 2x1", "few 3x1", "few 4x1", "256x256", "256x128", "128x128", "128x64", "64x64")

SOURCE = """
#include "choice.h"
extern "C" int way_of_q8(long long M, long long N, int cus) { return w4a8::q8_way(M, N, cus); }
extern "C" int ways_of_q8() { return w4a8::Q8_WAYS; }
extern "C" void way_of_ssm(long long B, long long T, long long NH, long long P, int N, int cus, int *way) {
  const w4a8::SsmWay w = w4a8::ssm_way(B, T, NH, P, N, cus);
  way[0] = w.rows, way[1] = w.single, way[2] = w.chunked, way[3] = w.slice;
}
"""


@functools.cache
def library():
    with tempfile.TemporaryDirectory() as d:
        src, so = os.path.join(d, "choice.cpp"), os.path.join(d, "choice.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-o", so, src,
                        "-I", os.path.join(ROOT, "paper_2606_24031_amd", "csrc")], check=True)
        L = ctypes.CDLL(so)
    I64, INT = ctypes.c_longlong, ctypes.c_int
    L.way_of_q8.argtypes = [I64, I64, INT]
    L.way_of_ssm.argtypes = [I64, I64, I64, I64, INT, INT, ctypes.POINTER(INT)]
    assert L.ways_of_q8() == len(Q8_WAYS)
    return L


def q8_way(M, N, cus):
    """The kernel of q8q8_gemm: channel tiles and row tiles of 16 of a wave, or
    channels and rows of a tile."""
    return Q8_WAYS[library().way_of_q8(M, N, cus)]


SsmWay = collections.namedtuple("SsmWay", "rows single chunked slice")


def ssm_way(B, T, NH, P, N, cus):
    """How ssm_scan takes a call: sequences of up to `rows` rows row by row (one
    at a time if `single`), the `chunked` longest by chunks, `slice` columns a
    workgroup."""
    way = (ctypes.c_int * 4)()
    library().way_of_ssm(B, T, NH, P, N, cus, way)
    return SsmWay(*way)
