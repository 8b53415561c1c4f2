"""How the tiles of the weights' gradient over experts are dealt to the work-groups of a launch, found out on the CPU: by eighths of every expert, or, where a 16-bit matrix is a few tiles along both sides, by
whole experts; every tile once in either way."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_06057_amd", "csrc")
F32, BF16 = 0, 1
ANY64, RING64, RING64X128 = 0, 5, 6

STUBS = """
#include "experts_host.h"
static int64_t g_seen[5];
static int g_ask = -1;
extern "C" long seen(int i) { return g_seen[i]; }
extern "C" void ask(int kernel) { g_ask = kernel; }
extern "C" int lcma_launch_experts_gemm(const lcma::ExpertsGemmParams *p, int, int kernel, int, int grid, void *) {
    g_seen[0] = kernel; g_seen[1] = grid; g_seen[2] = p->nx; g_seen[3] = p->nz; g_seen[4] = p->by_expert; return 0; }
extern "C" int lcma_launch_gated(const lcma::GatedParams *, int, int, int, int, void *) { return 0; }
namespace lcma {
lcma_status fail(lcma_status st, const char *, ...) { return st; }
int dtype_size(int d) { return d == 0 ? 4 : d == 1 || d == 2 ? 2 : 0; }
int tuning_experts_kernel() { return g_ask; }
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = tmp_path_factory.mktemp("deal")
    (out / "stubs.cc").write_text(STUBS)
    so = str(out / "deal.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(out / "stubs.cc"), os.path.join(CSRC, "experts_api.cc"), "-o", so])
    L = ctypes.CDLL(so)
    i64, vp, i32 = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
    L.seen.restype = ctypes.c_long
    L.lcma_gemm_experts_grad.argtypes = [i64, i64, i64, i32, vp, vp, i64, vp, i64, vp, i32, vp]
    return L


def gradient(L, kernel, rows, N, K, E, dtype=BF16):
    """grid, tiles along both sides, by experts or not"""
    L.ask(kernel)
    assert L.lcma_gemm_experts_grad(rows, N, K, E, 1 << 58, 1 << 59, N, 1 << 60, K, 1 << 61, dtype, None) == 0 and (kernel < 0 or L.seen(0) == kernel)
    return L.seen(1), L.seen(2), L.seen(3), bool(L.seen(4))


@pytest.mark.parametrize("kernel,dtype", [(RING64, BF16), (RING64X128, BF16), (RING64, F32), (ANY64, BF16)])
@pytest.mark.parametrize("N,K,E", [(304, 1104, 8), (384, 1152, 5), (160, 1408, 64), (64, 64, 7), (1000, 2000, 3), (64, 2048, 128), (512, 448, 1), (200, 320, 1000)])
def test_every_tile_once(lib, kernel, dtype, N, K, E):
    grid, nx, nz, by_expert = gradient(lib, kernel, 1000, N, K, E, dtype)
    of, jobs = nx * nz, E * nx * nz
    q = -(-jobs // 8) if by_expert else -(-of // 8)
    taken = sorted(job for b in range(grid) for job in [((b >> 3) // q * 8 + (b & 7)) * q + (b >> 3) % q] if job < jobs)
    assert taken == list(range(jobs))


def test_where_tiles_are_dealt_by_experts(lib):
    by_experts = lambda *a, **k: gradient(lib, *a, **k)[3]
    assert all(by_experts(k, 42342, 304, 1104, 8) for k in (RING64X128,)) and by_experts(-1, 42342, 304, 1104, 8) and by_experts(-1, 15360, 152, 1408, 8)
    assert not by_experts(RING64, 42342, 304, 1104, 8, dtype=F32) and not by_experts(ANY64, 42342, 304, 1104, 8)  # fp32, any sizes: by eighths
    assert not by_experts(RING64X128, 1000, 1000, 2000, 8)  # 16 x 16 tiles
    assert not by_experts(RING64X128, 1000, 2304, 184, 8) and not by_experts(RING64X128, 1000, 64, 1600, 8)  # long and narrow
    assert gradient(lib, RING64, 1000, 448, 448, 8)[1:] == (7, 7, True) and gradient(lib, RING64, 1000, 512, 512, 8)[1:] == (8, 8, False)
