"""Which kernel of the 8-bit-integer product a call runs, found out on the CPU with launchers that record instead of launching: the rule reaches every
kernel, launches cover all tiles and stay within the limits of a grid."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_06057_amd", "csrc")
NAMES = ["16x16", "32x32", "64x64", "64x128", "128x128", "128x256", "256x256"]

STUBS = """
#include "experts_host.h"
static int g_seen[4];
extern "C" int seen(int i) { return g_seen[i]; }
extern "C" int lcma_launch_i8_gemm(const lcma::I8GemmParams *p, int kernel, int, int grid, void *) {
    g_seen[0] = kernel; g_seen[1] = grid; g_seen[2] = p->nz; g_seen[3] = p->steps; return 0; }
extern "C" int lcma_launch_i8_quantize(const lcma::I8QuantParams *, int, int, int threads, void *) { g_seen[0] = threads; return 0; }
namespace lcma {
lcma_status fail(lcma_status st, const char *, ...) { return st; }
int dtype_size(int d) { return d == 0 ? 4 : d == 1 || d == 2 ? 2 : 0; }
int tuning_i8_kernel() { return -1; }
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = tmp_path_factory.mktemp("i8")
    stub = out / "stubs.cc"
    stub.write_text(STUBS)
    so = str(out / "i8.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(stub), os.path.join(CSRC, "i8_api.cc"), "-o", so])
    L = ctypes.CDLL(so)
    i64, vp = ctypes.c_int64, ctypes.c_void_p
    L.lcma_i8_gemm_nt.argtypes = [i64, i64, i64, vp, vp, vp, vp, vp, vp, i64, ctypes.c_int, vp]
    L.lcma_i8_gemm_experts.argtypes = [i64, i64, i64, ctypes.c_int, vp, vp, vp, vp, vp, vp, vp, i64, ctypes.c_int, vp]
    L.lcma_i8_quantize.argtypes = [i64, i64, vp, i64, ctypes.c_int, ctypes.c_int, vp, vp, vp]
    return L


def _dense(L, M, N, K):
    at = [1 << 44, 1 << 45, 1 << 46, 1 << 47, 1 << 50]
    assert L.lcma_i8_gemm_nt(M, N, K, at[0], at[1], at[2], at[3], None, at[4], N, 1, None) == 0
    return NAMES[L.seen(0)], L.seen(1)


def _experts(L, rows, N, K, E):
    at = [1 << 44, 1 << 45, 1 << 46, 1 << 47, 1 << 50, 1 << 51]
    assert L.lcma_i8_gemm_experts(rows, N, K, E, at[0], at[1], at[2], at[3], at[5], None, at[4], N, 1, None) == 0
    return NAMES[L.seen(0)], L.seen(1)


def test_every_kernel_is_reached(lib):
    shapes = [(1, 4096, 4096), (64, 4096, 4096), (256, 4096, 4096), (128, 14336, 4096), (1024, 4096, 4096), (2048, 4096, 4096), (8192, 14336, 4096)]
    assert [_dense(lib, *s)[0] for s in shapes] == NAMES
    got = {_experts(lib, rows, N, K, E)[0] for rows in (2, 16, 64, 300, 1500, 6000, 30000) for N, K in ((512, 1024), (2816, 2048), (28672, 4096)) for E in (8, 64, 128)}
    assert got >= {"16x16", "64x128", "128x256", "256x256"}


def test_launches_cover_every_tile(lib):
    for M, N, K in [(1, 1, 1), (1, 14336, 4096), (17, 65, 130), (300, 2000, 64), (8192, 100, 5000), (5000, 5000, 14336), (8192, 14336, 4096), (1 << 20, 64, 64)]:
        name, grid = _dense(lib, M, N, K)
        tm, tn = map(int, name.split("x"))
        tiles = -(-M // tm) * -(-N // tn)
        assert lib.seen(2) == -(-N // tn) and lib.seen(3) == -(-K // 128)
        if name in ("128x256", "256x256"):
            assert grid == min(tiles, 256)
        else:
            assert tiles <= grid < tiles + 8 and grid % 8 == 0
    for rows, N, K, E in [(1, 8, 8, 1024), (3, 100, 100, 8), (5000, 2816, 2048, 64), (70000, 500, 500, 3)]:
        name, grid = _experts(lib, rows, N, K, E)
        tm, tn = map(int, name.split("x"))
        # the most tiles that any split of the rows into groups can have: one row in each group but the last, or remainders of one row
        most = (rows // tm + min(rows, E)) * -(-N // tn)
        if name in ("128x256", "256x256"):
            assert grid == min(most, 256)
        else:
            assert grid >= most and grid % 8 == 0


def test_an_empty_k_takes_the_kernel_that_can(lib):
    assert _dense(lib, 8192, 14336, 0)[0] == "64x64"


def test_threads_of_a_row(lib):
    got = []
    for K in (1, 1024, 1025, 4096, 4097, 100000):
        assert lib.lcma_i8_quantize(10, K, 1 << 44, K, 1, 0, 1 << 45, 1 << 46, None) == 0
        got.append(lib.seen(0))
    assert got == [64, 64, 256, 256, 1024, 1024]
