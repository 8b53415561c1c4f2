"""Which kernel of the experts' products (in their own type and with 4-bit weights) and which launch of the gate a call runs, found out on the CPU with launchers that record instead of
launching: the rules reach every kernel, launches cover all tiles and stay within the limits of a grid, operands that a kernel does not hold go to one that does."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_06057_amd", "csrc")
NAMES = ["any64x64", "any128x128", "any32x32", "16x16", "32x32", "64x64", "64x128", "128x256", "256x256"]
NAMES4 = ["16x16", "16x32", "16x64", "64x64"]
F32, BF16, NT, NN, GRAD = 0, 1, 0, 1, 2
SHAPE = 5

STUBS = """
#include "experts_host.h"
static int64_t g_seen[8];
static int g_ask = -1;
extern "C" long seen(int i) { return g_seen[i]; }
extern "C" void ask(int kernel) { g_ask = kernel; }
extern "C" int lcma_launch_experts_gemm(const lcma::ExpertsGemmParams *p, int form, int kernel, int dtype, int grid, void *) {
    g_seen[0] = kernel; g_seen[1] = grid; g_seen[2] = p->nz; g_seen[3] = p->nx; g_seen[4] = form; g_seen[5] = dtype; g_seen[6] = p->stream; g_seen[7] = p->lines; return 0; }
extern "C" int lcma_launch_i4_gemm(const lcma::I4GemmParams *p, int kernel, int group, int dtype, int grid, void *) {
    g_seen[0] = kernel; g_seen[1] = grid; g_seen[2] = p->nz; g_seen[3] = group; g_seen[4] = p->blocks; g_seen[5] = dtype; return 0; }
extern "C" int lcma_launch_i4_prepare(const lcma::I4PrepareParams *, int dtype, int grid, void *) { g_seen[0] = dtype; g_seen[1] = grid; return 0; }
extern "C" int lcma_launch_gated(const lcma::GatedParams *p, int, int back, int gx, int gy, void *) {
    g_seen[0] = back; g_seen[1] = gx; g_seen[2] = gy; g_seen[3] = p->lane_shift; g_seen[4] = p->stream; return 0; }
namespace lcma {
lcma_status fail(lcma_status st, const char *, ...) { return st; }
int dtype_size(int d) { return d == 0 ? 4 : d == 1 || d == 2 ? 2 : 0; }
int tuning_experts_kernel() { return g_ask; }
int tuning_i4_kernel() { return g_ask < kI4Kernels ? g_ask : -1; }
}
"""


@pytest.fixture(scope="module")
def library(tmp_path_factory):
    out = tmp_path_factory.mktemp("experts")
    stub = out / "stubs.cc"
    stub.write_text(STUBS)
    so = str(out / "experts.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(stub)] + [os.path.join(CSRC, f) for f in ("experts_api.cc", "i4_api.cc")] + ["-o", so])
    L = ctypes.CDLL(so)
    i64, vp, i32 = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
    L.seen.restype = ctypes.c_long
    L.lcma_gemm_experts.argtypes = [i32, i64, i64, i64, i32, vp, vp, i64, vp, vp, i64, i32, vp]
    L.lcma_gemm_experts_grad.argtypes = [i64, i64, i64, i32, vp, vp, i64, vp, i64, vp, i32, vp]
    L.lcma_gated_silu.argtypes = [i64, i64, vp, i64, vp, i64, i32, vp]
    L.lcma_gated_silu_grad.argtypes = [i64, i64, vp, i64, vp, i64, vp, i64, i32, vp]
    L.lcma_i4_gemm_nt.argtypes = [i64, i64, i64, i32, vp, i64, vp, vp, vp, i64, i32, vp]
    L.lcma_i4_gemm_experts.argtypes = [i64, i64, i64, i32, i32, vp, vp, i64, vp, vp, vp, i64, i32, vp]
    L.lcma_i4_quantize.argtypes = [i32, i64, i64, i32, vp, i64, i32, vp, vp]
    return L


@pytest.fixture
def lib(library):
    library.ask(-1)
    return library


AT = [1 << 59, 1 << 60, 1 << 61, 1 << 62, 1 << 58]


def product(L, rows, N, K, E, form=NT, dtype=BF16, lda=None, ldc=None, a=0, w=0):
    """The kernel's name and the grid, or the status; a, w: bytes that A and the weights lie off 16."""
    st = L.lcma_gemm_experts(2 if form == NT else 0, rows, N, K, E, AT[4], AT[0] + a, lda or K, AT[1] + w, AT[2], ldc or N, dtype, None)
    return st or (NAMES[L.seen(0)], L.seen(1))


def gradient(L, rows, N, K, E, dtype=BF16, lda=None, lddc=None, a=0, d=0):
    st = L.lcma_gemm_experts_grad(rows, N, K, E, AT[4], AT[0] + d, lddc or N, AT[1] + a, lda or K, AT[2], dtype, None)
    return st or (NAMES[L.seen(0)], L.seen(1))


def four(L, rows, N, K, E=0, dtype=BF16, group=128):
    st = (L.lcma_i4_gemm_experts(rows, N, K, group, E, AT[4], AT[0], K, AT[1], None, AT[2], N, dtype, None) if E else
          L.lcma_i4_gemm_nt(rows, N, K, group, AT[0], K, AT[1], None, AT[2], N, dtype, None))
    return st or (NAMES4[L.seen(0)], L.seen(1))


def most_tiles(name, rows, N, E):
    """The most tiles that any split of the rows into groups can have: whole ones and one remainder for every expert that can have rows."""
    tm, tn = map(int, name.removeprefix("any").split("x"))
    return (rows // tm + min(rows, E)) * -(-N // tn)


def fits(name, grid, tiles, walking=("128x256", "256x256"), dealt=8):
    """dealt: the tiles that the work-groups are dealt in one go."""
    return grid == 256 if name in walking else tiles <= grid < tiles + dealt and grid % 8 == 0 and grid * 512 < 1 << 32


ROWS = (1, 2, 4, 8, 16, 32, 64, 100, 128, 250, 512, 1000, 2048, 4096, 16384)
SIZES = [(N, K, E) for N, K in ((256, 512), (512, 2048), (2816, 2048), (4096, 14336), (14336, 4096), (28672, 4096)) for E in (2, 8, 64, 128)]


def test_every_kernel_is_reached(lib):
    def seen(call, odd, **more):
        return {call(lib, rows, N - odd, K - odd, E, **more)[0] for rows in ROWS for N, K, E in SIZES}

    whole = {"16x16", "32x32", "64x64", "64x128", "128x256", "256x256"}
    assert seen(product, 0) == whole
    assert seen(product, 0, form=NN) == whole - {"16x16"}
    assert seen(gradient, 0) == {"64x64", "64x128", "256x256"}
    assert seen(product, 0, dtype=F32) == seen(product, 1, dtype=F32) == seen(product, 0, dtype=F32, form=NN) == {"32x32", "64x64"}
    assert seen(gradient, 0, dtype=F32) == {"any64x64", "64x64"}
    assert seen(product, 1) == {"any64x64", "any128x128", "any32x32"} and seen(product, 1, form=NN) == {"any64x64", "any32x32"}
    assert product(lib, 1, 1 << 28, 1, 64, form=NN) == ("any128x128", 1 << 21)  # more tiles of 64 columns than a launch holds
    assert seen(gradient, 1) == {"any64x64", "any128x128"}


def test_every_kernel_with_4_bit_weights_is_reached(lib):
    assert {four(lib, rows, N, K)[0] for rows in ROWS for N, K, _ in SIZES} == set(NAMES4)
    assert {four(lib, rows, N, K, E)[0] for rows in ROWS for N, K, E in SIZES} == set(NAMES4)
    assert {four(lib, rows, N, K, E, dtype=F32)[0] for rows in ROWS for N, K, E in SIZES} == set(NAMES4) - {"64x64"}


@pytest.mark.parametrize("ask", range(-1, len(NAMES)))
def test_launches_cover_every_tile(lib, ask):
    """By the rule, and with each kernel asked for by name, which calls that it does not hold ignore."""
    lib.ask(ask)
    for rows, N, K, E in [(1, 1, 1, 1), (1, 8, 8, 1024), (3, 100, 100, 8), (63, 65, 130, 64), (5000, 2816, 2048, 64), (70000, 500, 500, 3), (1 << 20, 64, 64, 2), (300, 1 << 20, 1024, 5)]:
        for dtype in (F32, BF16):
            for form in (NT, NN):
                name, grid = product(lib, rows, N, K, E, form, dtype)
                assert fits(name, grid, most_tiles(name, rows, N, E)) and lib.seen(4) == form
                assert lib.seen(2) == -(-N // int(name.split("x")[1]))
            name, grid = gradient(lib, rows, N, K, E, dtype)
            tm, tn = map(int, name.removeprefix("any").split("x"))
            of = -(-N // tm) * -(-K // tn)
            assert fits(name, grid, E * of, dealt=-(-of // 8) * 8) and lib.seen(4) == GRAD
            assert lib.seen(3) == -(-N // tm) and lib.seen(2) == -(-K // tn)


@pytest.mark.parametrize("ask", range(-1, len(NAMES4)))
def test_launches_with_4_bit_weights_cover_every_tile(lib, ask):
    lib.ask(ask)
    for rows, N, K, E in [(1, 1, 1, 1), (1, 8, 8, 1024), (3, 100, 100, 8), (5000, 2816, 2048, 64), (70000, 500, 500, 3), (1 << 20, 64, 64, 2)]:
        for dtype in (F32, BF16):
            name, grid = four(lib, rows, N, K, E, dtype)
            assert fits(name, grid, most_tiles(name, rows, N, E), ()) and lib.seen(2) == -(-N // int(name.split("x")[1])) and lib.seen(4) == -(-K // 128)
            name, grid = four(lib, rows, N, K, 0, dtype)
            tm, tn = map(int, name.split("x"))
            assert fits(name, grid, -(-rows // tm) * -(-N // tn), ())


@pytest.mark.parametrize("ask", range(-1, len(NAMES)))
def test_operands_off_whole_16_bytes_go_to_kernels_that_take_any(lib, ask):
    lib.ask(ask)
    for rows in (1, 100, 20000):
        ok = product(lib, rows, 512, 512, 8)[0]
        assert ask == -1 or ok == NAMES[ask]
        off = [product(lib, rows, 512, 512, 8, a=2), product(lib, rows, 512, 512, 8, w=8), product(lib, rows, 512, 511, 8, lda=512), product(lib, rows, 512, 512, 8, lda=513),
               product(lib, rows, 511, 512, 8, form=NN), product(lib, rows, 512, 512, 8, form=NN, w=2), gradient(lib, rows, 512, 512, 8, a=2), gradient(lib, rows, 512, 512, 8, d=2),
               gradient(lib, rows, 511, 512, 8), gradient(lib, rows, 512, 511, 8), gradient(lib, rows, 512, 512, 8, lda=514, lddc=512)]
        assert all(name.startswith("any") for name, _ in off)
        # N of weights N x K, K of weights K x N, and where the result lies, do not matter
        assert ask == -1 or NAMES[ask].startswith("any") or product(lib, rows, 511, 512, 8, ldc=511)[0] == NAMES[ask]
        assert not product(lib, rows, 512, 512, 8, ldc=513)[0].startswith("any") or ask in (0, 1, 2)
        # fp32 has kernels for any sizes alone
        assert product(lib, rows, 511, 333, 8, dtype=F32, lda=335, a=4, w=4)[0] == product(lib, rows, 511, 333, 8, dtype=F32)[0]


def test_gradients_that_pass_the_caches_by(lib):
    """In rows of whole 128-byte lines from such a line on; the largest tiles' waves write lines where an expert has up to 512 rows on average."""
    def of(rows, K, E, at=0, dtype=BF16):
        assert lib.lcma_gemm_experts_grad(rows, 512, K, E, AT[4], AT[0], 512, AT[1], K, AT[2] + at, dtype, None) == 0
        return bool(lib.seen(6)), bool(lib.seen(7))

    assert of(4096, 512, 8) == (True, True) and of(4097, 512, 8) == (True, False)
    assert of(100, 32, 8)[0] is False and of(100, 32, 8, dtype=F32)[0] is True and of(100, 520, 8)[0] is False and of(100, 512, 8, at=16)[0] is False


@pytest.mark.parametrize("ask", range(-1, len(NAMES)))
def test_rows_that_lie_far_apart_go_to_the_kernels_with_long_offsets(lib, ask):
    """The others' offsets inside a tile are 32-bit: rows of up to 2^22 bytes."""
    lib.ask(ask)
    long_offsets = {"any64x64", "any128x128"}
    far = 1 << 22  # elements: 2^23 bytes of 16 bit
    for rows in (1, 3000):
        for dtype in (F32, BF16):
            assert product(lib, rows, 64, 64, 4, lda=far, dtype=dtype)[0] in long_offsets
            assert product(lib, rows, 64, far, 4, dtype=dtype)[0] in long_offsets
            assert product(lib, rows, far, 64, 4, form=NN, dtype=dtype)[0] in long_offsets
            assert gradient(lib, rows, 64, 64, 4, lda=far, dtype=dtype)[0] in long_offsets
            assert gradient(lib, rows, 64, 64, 4, lddc=far, dtype=dtype)[0] in long_offsets
        assert product(lib, rows, 64, 64, 4, lda=far // 2)[0] not in long_offsets or ask in (0, 1)
        assert product(lib, rows, 64, 64, 4, ldc=far)[0] not in long_offsets or ask in (0, 1)
        assert product(lib, rows, 64, 0, 4)[0] in long_offsets  # nothing to sum


@pytest.mark.parametrize("ask", range(-1, len(NAMES)))
def test_more_tiles_than_any_launch_holds(lib, ask):
    lib.ask(ask)
    assert product(lib, (1 << 31) - 1, 1 << 20, 100, 2) == SHAPE
    assert product(lib, (1 << 31) - 1, 1 << 20, 100, 2, form=NN, dtype=F32) == SHAPE
    assert gradient(lib, 100, 1 << 21, 1 << 21, 1024) == SHAPE
    assert four(lib, (1 << 31) - 1, 1 << 20, 100) == four(lib, (1 << 31) - 1, 1 << 20, 100, 2) == SHAPE
    for rows, N, K in [(200000000, 1, 64), (1 << 27, 64, 64), (3, (1 << 27) - 1, 16)]:  # held by some kernels alone
        for name, grid in (product(lib, rows, N, K, 3), product(lib, rows, N, K, 3, dtype=F32)):
            assert fits(name, grid, most_tiles(name, rows, N, 3))


def test_gate(lib):
    """Threads along a row: a power of two of 8 columns each, up to 256; rows of up to 2^20 groups, which then take several; passing the caches from 64 MiB written."""
    for rows, F in [(1, 1), (2, 14336), (16384, 14336), (1 << 28, 8), (7, 100), ((1 << 31) - 1, 1)]:
        for back in (0, 1):
            st = (lib.lcma_gated_silu_grad(rows, F, AT[0], F, AT[1], 2 * F, AT[2], 2 * F, BF16, None) if back else
                  lib.lcma_gated_silu(rows, F, AT[0], 2 * F, AT[2], F, BF16, None))
            assert st == 0
            was_back, gx, gy, shift, stream = (lib.seen(i) for i in range(5))
            vectors = -(-F // 8)
            assert was_back == back and shift == min(8, (vectors - 1).bit_length()) and gy == -(-vectors // (1 << shift))
            assert gx == min(1 << 20, -(-rows // (256 >> shift))) and bool(stream) == (rows * F * 2 * (1 + back) >= 64 << 20)


def test_quantising_launches_at_most_65536_groups(lib):
    for E, N in [(1, 1), (8, 14336), (1024, 28672)]:
        assert lib.lcma_i4_quantize(E, N, 512, 128, AT[0], 512, BF16, AT[1], None) == 0
        assert lib.seen(1) == min(1 << 16, E * -(-N // 16))
