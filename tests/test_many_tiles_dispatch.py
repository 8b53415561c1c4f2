"""Products with more tiles than one launch has work-groups for, of sizes that a GPU's memory holds: several launches, which cover every tile once and each stay within the limits of a grid.  Found
out on the CPU with launchers that record instead of launching."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_06057_amd", "csrc")
F32, BF16 = 0, 1
TILES4 = [(16, 16), (16, 32), (16, 64), (64, 64)]

STUBS = """
#include "experts_host.h"
#include <vector>
static std::vector<int64_t> g_seen; // kernel, from, grid of every launch
extern "C" long seen(long i) { return i < (long)g_seen.size() ? g_seen[i] : -1; }
extern "C" void clear() { g_seen.clear(); }
template <class P> static int note(const P *p, int kernel, int grid) { for (int64_t v : {(int64_t)kernel, (int64_t)p->from, (int64_t)grid}) g_seen.push_back(v); return 0; }
extern "C" int lcma_launch_i4_gemm(const lcma::I4GemmParams *p, int kernel, int, int, int grid, void *) { return note(p, kernel, grid); }
extern "C" int lcma_launch_experts_gemm(const lcma::ExpertsGemmParams *p, int, int kernel, int, int grid, void *) { return note(p, kernel, grid); }
extern "C" int lcma_launch_gated(const lcma::GatedParams *, int, int, int, int, void *) { return 0; }
extern "C" int lcma_launch_i4_prepare(const lcma::I4PrepareParams *, int, int, void *) { return 0; }
namespace lcma {
lcma_status fail(lcma_status st, const char *, ...) { return st; }
int dtype_size(int d) { return d == 0 ? 4 : d == 1 || d == 2 ? 2 : 0; }
int tuning_i4_kernel() { return -1; }
int tuning_experts_kernel() { return -1; }
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = tmp_path_factory.mktemp("many_tiles")
    (out / "stubs.cc").write_text(STUBS)
    so = str(out / "many.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(out / "stubs.cc"), os.path.join(CSRC, "i4_api.cc"), os.path.join(CSRC, "experts_api.cc"), "-o", so])
    L = ctypes.CDLL(so)
    i64, vp, i32 = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
    L.seen.restype, L.seen.argtypes = ctypes.c_long, [ctypes.c_long]
    L.lcma_gemm_experts.argtypes = [i32, i64, i64, i64, i32, vp, vp, i64, vp, vp, i64, i32, vp]
    L.lcma_gemm_experts_grad.argtypes = [i64, i64, i64, i32, vp, vp, i64, vp, i64, vp, i32, vp]
    L.lcma_i4_gemm_nt.argtypes = [i64, i64, i64, i32, vp, i64, vp, vp, vp, i64, i32, vp]
    L.lcma_i4_gemm_experts.argtypes = [i64, i64, i64, i32, i32, vp, vp, i64, vp, vp, vp, i64, i32, vp]
    return L


AT = [1 << 59, 1 << 60, 1 << 61, 1 << 62, 1 << 58]


def launches(L, call, *args):
    """The kernel and [(from, grid)] of a call."""
    L.clear()
    assert getattr(L, call)(*args) == 0
    seen = []
    while L.seen(len(seen)) >= 0:
        seen.append(L.seen(len(seen)))
    kernels = set(seen[::3])
    assert len(kernels) == 1
    return kernels.pop(), list(zip(seen[1::3], seen[2::3]))


def covered(parts, eighth):
    """Work-group b of a launch takes tile from + b // 8 of the eighth b % 8: whether the launches take each of an eighth's tiles once, within 2^31 threads (512 a work-group)."""
    at = 0
    for start, grid in parts:
        assert start == at and grid % 8 == 0 and 0 < grid * 512 < 1 << 31
        at += grid // 8
    return at >= eighth and at - eighth < 8


# rows, N, K, type: 16 and 32 GB of C; a column; as many tiles as one launch just holds, and one more
CALLS4 = [(1 << 20, 4096, 64, F32), (1 << 20, 16384, 64, BF16), (1 << 22, 4096, 64, BF16), ((1 << 28) + 100, 1, 1, BF16), ((1 << 26) + 100, 1, 1, F32), ((1 << 31) - 1, 1, 1, BF16),
          (((1 << 22) - 9) * 16, 64, 64, F32), (((1 << 22) - 8) * 16, 64, 64, F32)]


@pytest.mark.parametrize("experts", [0, 1, 1000])
@pytest.mark.parametrize("rows,N,K,dtype", CALLS4)
def test_4_bit_weights(lib, rows, N, K, dtype, experts):
    args = (rows, N, K, 64) + ((experts, AT[4]) if experts else ()) + (AT[0], K, AT[1], None, AT[2], N, dtype, None)
    kernel, parts = launches(lib, "lcma_i4_gemm_experts" if experts else "lcma_i4_gemm_nt", *args)
    tm, tn = TILES4[kernel]
    tiles = (rows // tm + min(rows, experts) if experts else -(-rows // tm)) * -(-N // tn)
    assert covered(parts, -(-tiles // 8))
    assert dtype == BF16 or kernel != 3


def test_one_launch_where_it_holds_all_tiles(lib):
    for rows in (1, 1000, ((1 << 22) - 9) * 16):
        assert len(launches(lib, "lcma_i4_gemm_nt", rows, 64, 64, 64, AT[0], 64, AT[1], None, AT[2], 64, F32, None)[1]) == 1


ANY128 = 1  # the kernel with the fewest tiles of those for any sizes


@pytest.mark.parametrize("layout", [0, 2])
@pytest.mark.parametrize("rows,N,K,E,dtype", [((1 << 29) + 1000, 1, 1, 3, F32), ((1 << 29) + 1000, 1, 1, 3, BF16), (1 << 30, 8, 7, 1024, BF16), (1 << 30, 8, 8, 2, F32), ((1 << 31) - 1, 1, 1, 1, F32),
                                              (3, (1 << 29) - 1, 7, 1, BF16), (3, (1 << 29) - 1, 7, 2, F32)])
def test_experts_products(lib, rows, N, K, E, dtype, layout):
    kernel, parts = launches(lib, "lcma_gemm_experts", layout, rows, N, K, E, AT[4], AT[0], K, AT[1], AT[2], N, dtype, None)
    assert kernel == ANY128 and len(parts) > 1 and covered(parts, -(-(rows // 128 + min(rows, E)) * -(-N // 128) // 8))


@pytest.mark.parametrize("rows,N,K,E,dtype", [(2, 1, (1 << 29) - 1, 1, BF16), (2, (1 << 29) - 1, 1, 2, F32), (5, 3, (1 << 25) + 1, 1024, BF16), (5, 100, 12800, 1024, F32), (9, (1 << 21) + 1, 1024, 33, F32)])
def test_weights_gradients(lib, rows, N, K, E, dtype):
    """The kernels take, of every expert in turn, the eight eighths of its tiles (each rounded up)."""
    kernel, parts = launches(lib, "lcma_gemm_experts_grad", rows, N, K, E, AT[4], AT[0], N, AT[1], K, AT[2], dtype, None)
    tm = (64, 128)[kernel] if kernel < 2 else 64
    eighth = -(-(-(-N // tm) * -(-K // tm)) // 8)
    tiles = E * -(-N // tm) * -(-K // tm)
    assert covered(parts, -(-tiles // (8 * eighth)) * eighth)
    assert (len(parts) > 1) == (tiles + 8 >= 1 << 22) and (kernel == ANY128 or len(parts) == 1)
