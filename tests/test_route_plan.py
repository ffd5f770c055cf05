"""Workspace of the router's gradient, on the CPU: no token count needs more than it is given, and a context is not asked for more than its
FFN's workspace while that holds the partial sums.  csrc/route_plan.hpp is compiled here as plain C++."""
import ctypes
import os
import subprocess

import pytest

from paper_2411_16786_amd import binding as B

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2411_16786_amd", "csrc")
SHIM = """#include "route_plan.hpp"
// the first T up to T_max whose chunks are more than the bound for T tokens, 0 if there is none
extern "C" int beyond(int T_max, int E, int columns) {
    for (int T = 1; T <= T_max; ++T) {
        const int chunk = dicemoe::route_chunk(T, E, columns);
        if ((T + chunk - 1) / chunk > dicemoe::route_chunks_most(T, E, columns)) return T;
        if (dicemoe::route_chunks_most(T, E, columns) < dicemoe::route_chunks_most(T - 1, E, columns)) return T;
    }
    return 0;
}
extern "C" long long most(int T_max, int E, int columns) { return dicemoe::route_chunks_most(T_max, E, columns); }
extern "C" int chunk(int T, int E, int columns) { return dicemoe::route_chunk(T, E, columns); }
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    folder = tmp_path_factory.mktemp("route_plan")
    src, out = folder / "plan.cpp", folder / "plan.so"
    src.write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, str(src), "-o", str(out)], check=True)
    L = ctypes.CDLL(str(out))
    L.most.restype = ctypes.c_longlong
    return L


@pytest.mark.parametrize("E", [8, 33])
def test_no_token_count_has_more_chunks_than_the_bound(plan, E):
    for columns in [*range(1, 40), 63, 64, 65, 127, 128, 255, 256, 257, 512, 1000, 8192]:
        assert plan.beyond(70000, E, columns) == 0, columns


def test_chunks_are_as_measured(plan):
    assert [plan.chunk(T, 16, 16) for T in (1, 2048, 4096, 8192)] == [64, 64, 128, 256]
    assert plan.most(8192, 16, 16) == 32 and plan.most(1 << 20, 16, 16) == 4096 and plan.most(10, 16, 16) == 1


def _ffn_bytes(T_max, d, F, k, dtype, E):
    """Hidden activations, partial sums of a split second GEMM, status words; the dispatch's scratch is smaller here."""
    hidden = (T_max * k * F * (2 if dtype == "bf16" else 4) + 255) // 256 * 256
    return hidden + (288 * 128 * 192 * 4 if dtype == "bf16" else 0) + 4096


@pytest.mark.parametrize("shape", [(8192, 2048, 256, 16, 1, "bf16"), (8192, 1024, 64, 64, 2, "bf16"), (4096, 1152, 4608, 8, 2, "bf16"), (4096, 384, 1536, 16, 2, "f32"),
                                   (8192, 2048, 8192, 16, 2, "bf16")])
def test_the_router_gradient_needs_no_workspace_of_its_own(shape):
    T_max, d, F, E, k, dtype = shape
    assert B.Context(T_max, d, F, E, k, dtype).workspace_bytes() == _ffn_bytes(T_max, d, F, k, dtype, E)


@pytest.mark.parametrize("shape", [(8192, 4096, 64, 64, 1, "bf16"), (8192, 4096, 16, 64, 1, "f32"), (64, 64, 64, 64, 1, "f32")])
def test_where_it_needs_more_it_gets_it(plan, shape):
    T_max, d, F, E, k, dtype = shape
    columns = -(-d // (128 if dtype == "bf16" else 64))
    need = 4 * (plan.most(T_max, E, columns) * E * (d + 1) + T_max * E)
    have = B.Context(T_max, d, F, E, k, dtype).workspace_bytes()
    assert have >= need + 4096 and have == max(_ffn_bytes(T_max, d, F, k, dtype, E), (need + 255) // 256 * 256 + 4096)
