"""The rule of csrc/matmul_i8_plan.h, compiled for the host: how a product is cut, without a GPU; and products of every kind."""
import ctypes
import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2508_12851_amd", "csrc")
TILES = {"64x64": (64, 64), "64x128": (64, 128), "128x128": (128, 128), "256x256": (256, 256), "short": (128, 128)}

_SOURCE = """
#include "matmul_i8_plan.h"
extern "C" int plan(int M, int N, int K) {
  const prism::mm8::Plan p = prism::mm8::plan_of(M, N, K);
  return (int)p.tile * 100 + p.splits;
}
"""


@functools.lru_cache(maxsize=1)
def _lib():
    d = tempfile.mkdtemp(prefix="matmul_plans_")
    src, so = os.path.join(d, "p.cpp"), os.path.join(d, "p.so")
    with open(src, "w") as f:
        f.write(_SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, "-I", os.path.join(ROOT, "include"), src, "-o", so],
                   check=True, timeout=120)
    return ctypes.CDLL(so)


def plan(m, n, k):
    """(tile, splits of the contraction) of a product of m rows, n columns and k elements each."""
    v = _lib().plan(m, n, k)
    return list(TILES)[v // 100], v % 100


# Products that take every tile, with and without splits, and what they take: m, n, k, tile, splits.
PRODUCTS = [
    (4100, 4099, 130, "short", 1), (77, 2053, 1411, "64x64", 1), (200, 3000, 4096, "64x64", 1), (1, 5466, 3482, "64x64", 2), (1, 4545, 2596, "64x64", 3),
    (3, 3999, 4096, "64x64", 4), (64, 128, 8192, "64x64", 8), (139, 5808, 265, "64x128", 1), (500, 2201, 1411, "64x128", 1),
    (77, 3229, 4463, "64x128", 4), (66, 2786, 3680, "64x128", 5), (65, 2138, 4348, "64x128", 6), (2101, 68, 4248, "64x128", 7),
    (70, 1650, 6724, "64x128", 8), (600, 4096, 2048, "128x128", 1), (1119, 2189, 449, "128x128", 1), (136, 5582, 15153, "128x128", 2),
    (66, 5395, 5610, "128x128", 4), (1603, 132, 13964, "128x128", 8), (2048, 8192, 512, "256x256", 1), (2443, 1666, 260, "256x256", 1),
    (2950, 1557, 409, "256x256", 1),
]
