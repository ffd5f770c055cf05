"""The tile rule of the 4-bit expert FFN (csrc/mx4_plan.hpp, compiled here as plain C++).  Needs no GPU."""
import ctypes
import functools
import os
import subprocess
import tempfile

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2411_16786_amd", "csrc")
SHIM = """#include "mx4_plan.hpp"
extern "C" int tile(int rows, int n_seg, int N, int K) { return dicemoe::pick_tile(rows, n_seg, N, K); }
extern "C" int chunks(int tile, int K) { return dicemoe::tile_chunks(tile, K) ? 1 : 0; }
extern "C" int lds(int tile, int K) { return dicemoe::tile_lds(tile, K, dicemoe::tile_chunks(tile, K)); }
extern "C" int narrow(int rows, int n_seg, int N) { return dicemoe::rows_narrow(rows, n_seg, N) ? 1 : 0; }
extern "C" int wide(int rows, int n_seg, int N) { return dicemoe::rows_wide(rows, n_seg, N) ? 1 : 0; }
extern "C" int tile_t(int rows, int n_seg, int K) { return dicemoe::pick_tile_t(rows, n_seg, K); }
extern "C" long long bound(int rows, int n_seg, int BM) { return dicemoe::tile_bound(rows, n_seg, BM); }
"""
TILES = ["128x256", "128x128", "64x128", "32x128/2", "32x64/4", "64x128/2"]
TILES_T = ["64x256", "32x128/2", "32x128/4"]


@functools.lru_cache(None)
def lib():
    with tempfile.TemporaryDirectory(prefix="mx4_plan_") as folder:
        src, out = os.path.join(folder, "plan.cpp"), os.path.join(folder, "plan.so")
        with open(src, "w") as f:
            f.write(SHIM)
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, src, "-o", out], check=True)
        L = ctypes.CDLL(out)
        L.bound.restype = ctypes.c_longlong
        return L


def plan(rows, n_seg, N, K):
    """Kernel of a forward product to N columns over K: a tile, "+" behind it with scales by chunks, or the width of rows in sixteens."""
    t = lib().tile(rows, n_seg, N, K)
    if t < 0:
        return "rows16" if lib().narrow(rows, n_seg, N) else "rows32"
    return TILES[t] + ("+" if lib().chunks(t, K) else "")


def plan_float(rows, n_seg, N):
    return "rows64" if lib().wide(rows, n_seg, N) else "rows16" if lib().narrow(rows, n_seg, N) else "rows32"


def plan_t(rows, n_seg, K):
    t = lib().tile_t(rows, n_seg, K)
    return "rows" if t < 0 else TILES_T[t]


def plans(rows, n_seg, d, F):
    """Of the forward's two products and of the gradient's two."""
    return plan(rows, n_seg, F, d), plan(rows, n_seg, d, F), plan_t(rows, n_seg, F), plan_t(rows, n_seg, d)


def columns_left(kernel, N):
    """Columns of N behind the last whole block of a kernel, by its name."""
    block = {"rows16": 16, "rows32": 32, "rows64": 64, "rows": 128}.get(kernel)
    return N % (block or int(kernel.rstrip("+").split("/")[0].split("x")[1]))
