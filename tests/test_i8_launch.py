"""What a call of the 8-bit-integer product launches, found out on the CPU with launchers that record instead of launching: sizes that some kernels' launches do not
hold, kernels asked for by name, the grids of the kernels whose work-groups walk through tiles."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_06057_amd", "csrc")
GEN = os.path.join(CSRC, "generated")
NAMES = ["16x16", "32x32", "64x64", "64x128", "128x128", "128x256", "256x256"]

# (the library's own host side for the settings; other launchers stay unresolved, none is reached)
STUBS = """
#include "experts_host.h"
static int g_seen[4];
extern "C" int seen(int i) { return g_seen[i]; }
extern "C" int lcma_launch_i8_gemm(const lcma::I8GemmParams *p, int kernel, int, int grid, void *) {
    g_seen[0] = kernel; g_seen[1] = grid; g_seen[2] = p->nz; g_seen[3] = p->steps; return 0; }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if not os.path.exists(os.path.join(GEN, "registry.cc")):
        from paper_2605_06057_amd.gen.generate import generate
        generate(GEN)
    out = tmp_path_factory.mktemp("i8")
    stub = out / "stubs.cc"
    stub.write_text(STUBS)
    so = str(out / "i8.so")
    host = [os.path.join(CSRC, f) for f in ("i8_api.cc", "api.cc", "scheme.cc", "model.cc", "unfused.cc", "fp8_api.cc", "plane_gemm.cc")]
    missing = out / "missing.cc"
    flags = ["g++", "-std=c++17", "-O1", "-fPIC", "-I", CSRC, "-I", GEN]
    subprocess.check_call(flags + ["-shared", "-Wl,-Bsymbolic", str(stub)] + host + ["-o", so])
    # kernels' launchers and tables that this library does not hold: an address that nothing calls
    names = {line.split()[-1] for line in subprocess.check_output(["nm", "-D", "-u", so], text=True).splitlines()}
    names = {n for n in names if n.startswith("lcma_launch") or n.startswith("_ZN4lcma")}
    missing.write_text("".join(f'extern "C" {{ long {n}[16]; }}\n' for n in sorted(names)))
    subprocess.check_call(flags + ["-shared", "-Wl,-Bsymbolic", str(stub), str(missing)] + host + ["-o", so])
    L = ctypes.CDLL(so)
    i64, vp = ctypes.c_int64, ctypes.c_void_p
    L.lcma_i8_gemm_nt.argtypes = [i64, i64, i64, vp, vp, vp, vp, vp, vp, i64, ctypes.c_int, vp]
    L.lcma_i8_gemm_experts.argtypes = [i64, i64, i64, ctypes.c_int, vp, vp, vp, vp, vp, vp, vp, i64, ctypes.c_int, vp]
    yield L
    L.lcma_set_tuning(b"i8_kernel", b"")


AT = [1 << 54, 1 << 55, 1 << 56, 1 << 57, 1 << 60, 1 << 59]


def _dense(L, M, N, K):
    return L.lcma_i8_gemm_nt(M, N, K, AT[0], AT[1], AT[2], AT[3], None, AT[4], N, 1, None) or (NAMES[L.seen(0)], L.seen(1))


def _experts(L, rows, N, K, E):
    return L.lcma_i8_gemm_experts(rows, N, K, E, AT[0], AT[1], AT[2], AT[3], AT[5], None, AT[4], N, 1, None) or (NAMES[L.seen(0)], L.seen(1))


def _fits(name, grid, tiles):
    return grid == 256 if name in ("128x256", "256x256") else tiles <= grid < tiles + 8 and grid % 8 == 0 and grid * 512 < 1 << 31


@pytest.mark.parametrize("M,N,K", [(300000000, 1, 64), (269000000, 64, 128), ((1 << 31) - 1, 1, 64), (1 << 30, 700, 100), (300000000, 1, 0), ((1 << 31) - 1, 1, 0), (1, (1 << 29) - 1, 64), (70000, 1 << 20, 0)])
def test_sizes_that_some_launches_do_not_hold(lib, M, N, K):
    for name, grid, tiles in [(*_dense(lib, M, N, K), lambda tm: -(-M // tm)), (*_experts(lib, M, N, K, 3), lambda tm: M // tm + min(M, 3))]:
        tm, tn = map(int, name.split("x"))
        assert _fits(name, grid, tiles(tm) * -(-N // tn)) and lib.seen(2) == -(-N // tn)


def test_more_tiles_than_any_launch_holds(lib):
    assert _dense(lib, (1 << 31) - 1, 1 << 20, 100) == 5  # SHAPE
    assert _dense(lib, (1 << 31) - 1, 1 << 20, 0) == 5


@pytest.mark.parametrize("M,N,K", [(512, 14336, 4096), (1000, 1000, 1000), (2049, 2304, 257)])
def test_walking_kernels_launch_a_work_group_for_every_compute_unit(lib, M, N, K):
    """Also where there are fewer tiles: half a tile each for up to 128 of 256 x 256, and the rows behind the groups are shared by all."""
    for kernel in (b"128x256", b"256x256"):
        assert lib.lcma_set_tuning(b"i8_kernel", kernel) == 0
        assert _dense(lib, M, N, K) == (kernel.decode(), 256) == _experts(lib, M, N, K, 4)
    lib.lcma_set_tuning(b"i8_kernel", b"")


def test_kernels_by_name(lib):
    rule = _dense(lib, 333, 4096, 4096)
    for name in NAMES:
        lib.lcma_set_tuning(b"i8_kernel", name.encode())
        assert _dense(lib, 333, 4096, 4096)[0] == name
    for other in (b"7x9", b"64", b""):
        lib.lcma_set_tuning(b"i8_kernel", b"16x16")
        lib.lcma_set_tuning(b"i8_kernel", other)
        assert _dense(lib, 333, 4096, 4096) == rule
    lib.lcma_set_tuning(b"i8_kernel", b"16x16")  # (2^26 tiles: more than its launch holds)
    assert _dense(lib, 1 << 30, 1, 64)[0] in ("128x256", "256x256")
    lib.lcma_set_tuning(b"i8_kernel", b"")


def test_work_groups_of_a_launch(tmp_path):
    """Two dimensions hold any number of work-groups of up to 1024 threads, and few more than that."""
    src = tmp_path / "groups.cc"
    src.write_text('#include "lcma_experts_params.h"\nextern "C" long groups(long n, int which) { return which ? lcma::groups_of(n).across : lcma::groups_of(n).along; }\n')
    so = str(tmp_path / "groups.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(src), "-o", so])
    f = ctypes.CDLL(so).groups
    f.argtypes, f.restype = [ctypes.c_long, ctypes.c_int], ctypes.c_long
    for n in (1, 255, (1 << 20) - 1, 1 << 20, (1 << 20) + 1, (1 << 22) + 5, (1 << 24) + 1, (1 << 31) - 1):
        along, across = f(n, 0), f(n, 1)
        assert along * across >= n > along * (across - 1) and along * 1024 < 1 << 32 and across <= 65535 and (across == 1 or n > 1 << 20)
