"""lcma_gemm_experts and lcma_gemm_experts_grad against the products of each expert in 64 bits.

Whole numbers: inputs are -4 .. 4 and sums stay below 2^24, so every fp32 sum is exact and C is the exact result rounded once: no tolerance.
Real numbers: products of 16-bit inputs are exact in fp32, and every fp32 addition is off by at most 2^-23 of a partial sum (rounded or cut off), so a sum over k by
k 2^-23 sum |a b| (fp32 inputs: products are rounded too, 2 k 2^-23); rounding adds half a step of C's type (below its smallest normal number, fp16 2^-14, a step is
that number's: 2^-24)."""
import numpy as np
import pytest

from oracle import experts as X

pytestmark = pytest.mark.gpu
TYPES = ["bf16", "f16", "f32"]


def _torch():
    import torch
    return torch, {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _lib():
    from paper_2605_06057_amd import binding
    return binding


@pytest.fixture(params=["", "any64x64", "any128x128", "any32x32", "16x16", "32x32", "64x64", "64x128", "128x256", "256x256"], scope="module")
def kernel(request):
    """The kernel of the rule, and every kernel by name where it takes the sizes."""
    _lib().lcma_set_tuning("experts_kernel", request.param)
    yield request.param
    _lib().lcma_set_tuning("experts_kernel", "")


def _offsets(counts):
    torch, _ = _torch()
    return torch.tensor(np.cumsum([0] + list(counts)), dtype=torch.int32, device="cuda")


def _whole(gen, *shape):
    torch, _ = _torch()
    return torch.randint(-4, 5, shape, device="cuda", generator=gen).float()


def _normal(gen, *shape):
    torch, _ = _torch()
    return torch.randn(shape, device="cuda", generator=gen)


def _padded(t, pad, fill):
    """t as the left part of a wider tensor, whose other columns hold `fill`."""
    torch, _ = _torch()
    wide = torch.full((t.shape[0], t.shape[1] + pad), fill, dtype=t.dtype, device="cuda")
    wide[:, : t.shape[1]] = t
    return wide, wide[:, : t.shape[1]]


def _np(t):
    return t.double().cpu().numpy()


def _rounded(c, t):
    """A 64-bit result rounded once to type t (exact sums are fp32 numbers, so rounding by way of fp32 is one rounding)."""
    torch, types = _torch()
    return torch.from_numpy(c).float().to(types[t]).double().numpy()


COUNTS = [
    [1], [0, 3, 0, 0, 1], [2, 1], [17, 0, 33, 64], [65, 63, 1, 130], [5] * 70 + [0] * 60 + [3], [300, 0, 257, 9], [0, 0, 0],
]


@pytest.mark.parametrize("b_nk", [True, False])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: f"{sum(c)}of{len(c)}")
@pytest.mark.parametrize("N,K,pad,behind", [(64, 64, 0, 0), (1, 1, 0, 2), (8, 200, 8, 1), (130, 72, 0, 5), (200, 136, 16, 0), (33, 77, 3, 40)])
def test_product_of_whole_numbers(kernel, counts, N, K, pad, behind, dtype, b_nk):
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(sum(counts) + N)
    E, rows = len(counts), sum(counts) + behind
    a, w = _whole(gen, rows, K).to(types[dtype]), _whole(gen, E, *((N, K) if b_nk else (K, N))).to(types[dtype])
    _, av = _padded(a, pad, float("nan"))
    if behind:
        av[sum(counts):] = float("nan")  # (rows of no expert are not read)
    wide, c = _padded(torch.full((rows, N), 99.0, device="cuda").to(types[dtype]), pad, 7.0)
    offsets = _offsets(counts)
    assert _lib().lcma_gemm_experts(av, offsets, w, c, b_nk) is c
    want = X.gemm_experts(np.nan_to_num(_np(av)), offsets.cpu().numpy(), _np(w), b_nk)
    want[sum(counts):] = 0
    assert np.array_equal(_np(c), _rounded(want, dtype))
    assert (wide[:, N:] == 7.0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: f"{sum(c)}of{len(c)}")
@pytest.mark.parametrize("N,K,pad,behind", [(64, 64, 0, 0), (1, 1, 0, 2), (8, 200, 8, 1), (130, 72, 0, 5), (200, 136, 16, 0), (33, 77, 3, 40)])
def test_gradient_of_whole_numbers(kernel, counts, N, K, pad, behind, dtype):
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(sum(counts) + N)
    E, rows = len(counts), sum(counts) + behind
    _, dc = _padded(_whole(gen, rows, N).to(types[dtype]), pad, float("nan"))
    _, a = _padded(_whole(gen, rows, K).to(types[dtype]), pad, float("nan"))
    if behind:
        dc[sum(counts):] = float("nan")
        a[sum(counts):] = float("inf")
    dw = torch.full((E + 2, N, K), 99.0, device="cuda").to(types[dtype])
    offsets = _offsets(counts)
    _lib().lcma_gemm_experts_grad(dc, a, offsets, dw[1:-1])
    kept = slice(0, sum(counts))
    want = X.gemm_experts_grad(_np(dc[kept]), _np(a[kept]), offsets.cpu().numpy())
    assert np.array_equal(_np(dw[1:-1]), _rounded(want, dtype))
    assert (dw[0] == 99.0).all() and (dw[-1] == 99.0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("off", [0, 8, 32])
@pytest.mark.parametrize("counts", [[1], [0, 40, 300], [1500, 100]], ids=lambda c: f"{sum(c)}of{len(c)}")
@pytest.mark.parametrize("N,K", [(300, 320), (512, 576), (256, 256), (257, 1024), (70, 64)])
def test_gradient_in_rows_of_whole_lines(kernel, N, K, counts, off, dtype):
    """Rows of 128, 512, ... bytes from a multiple of 128 on or not: what is written past the caches and what is not, with many rows an expert and with few."""
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(N + K + off)
    E, rows = len(counts), sum(counts)
    dc, a = _whole(gen, rows, N).to(types[dtype]), _whole(gen, rows, K).to(types[dtype])
    room = torch.full((E * N * K + off + 64,), 99.0, device="cuda").to(types[dtype])
    dw = room[off:off + E * N * K].view(E, N, K)
    offsets = _offsets(counts)
    _lib().lcma_gemm_experts_grad(dc, a, offsets, dw)
    assert np.array_equal(_np(dw), _rounded(X.gemm_experts_grad(_np(dc), _np(a), offsets.cpu().numpy()), dtype))
    assert (room[:off] == 99.0).all() and (room[off + E * N * K:] == 99.0).all()


def _close(got, want, magnitude, k, dtype):
    torch, types = _torch()
    f = torch.finfo(types[dtype])
    step = 0 if dtype == "f32" else f.eps / 2
    tolerance = (2 if dtype == "f32" else 1) * k * 2.0 ** -23 * magnitude * (1 + step) + step * np.maximum(np.abs(want), f.smallest_normal)
    assert (np.abs(got - want) <= tolerance).all(), float((np.abs(got - want) - tolerance).max())


# rows of experts, N, K: a token's, short prompts, larger tiles, long sums, several tiles along every side
REAL = [([1, 0, 1, 0], 520, 1032), ([3, 2, 0, 5, 1, 4], 264, 2056), ([100, 90, 120, 70], 328, 520), ([1000, 300], 520, 264), ([700, 0, 900, 513], 1032, 584),
        ([2100, 1900], 776, 320), ([33, 700], 257, 131)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("counts,N,K", REAL, ids=str)
def test_real_numbers_and_both_gradients(kernel, counts, N, K, dtype):
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(N + K)
    E, rows = len(counts), sum(counts)
    a, w, dc = (_normal(gen, *s).to(types[dtype]) for s in ((rows, K), (E, N, K), (rows, N)))
    offsets = _offsets(counts)
    L = _lib()
    c, da, dw = L.lcma_gemm_experts(a, offsets, w), L.lcma_gemm_experts(dc, offsets, w, b_nk=False), L.lcma_gemm_experts_grad(dc, a, offsets)
    assert c.shape == (rows, N) and da.shape == a.shape and dw.shape == w.shape and c.dtype == da.dtype == dw.dtype == types[dtype]
    o, an, wn, dcn = offsets.cpu().numpy(), _np(a), _np(w), _np(dc)
    _close(_np(c), X.gemm_experts(an, o, wn), X.gemm_experts(np.abs(an), o, np.abs(wn)), K, dtype)
    _close(_np(da), X.gemm_experts(dcn, o, wn, False), X.gemm_experts(np.abs(dcn), o, np.abs(wn), False), N, dtype)
    _close(_np(dw), X.gemm_experts_grad(dcn, an, o), X.gemm_experts_grad(np.abs(dcn), np.abs(an), o), max(counts), dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_against_differences(dtype):
    """sum(C * up) is linear in A and in W: a step of 1 in one element changes it by the gradient, exactly in whole numbers."""
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(3)
    counts, N, K = [5, 0, 9, 20], 24, 40
    a, w, up = (_whole(gen, *s).to(types[dtype]) for s in ((34, K), (4, N, K), (34, N)))
    offsets, L = _offsets(counts), _lib()
    value = lambda a_, w_: (_np(L.lcma_gemm_experts(a_, offsets, w_)) * _np(up)).sum()
    da, dw = _np(L.lcma_gemm_experts(up, offsets, w, b_nk=False)), _np(L.lcma_gemm_experts_grad(up, a, offsets))
    # (results of up to 40 * 16 = 640: above 256 bf16 numbers are 2 or 4 apart, so a difference is off by up to 2 * 2 * the sum of |up|, fp32 and fp16: by nothing)
    slack = 4 * 4 * N if dtype == "bf16" else 0
    for r, k in [(0, 0), (4, 39), (5, 7), (33, 20)]:
        b = a.clone()
        b[r, k] += 1
        assert abs(value(b, w) - value(a, w) - da[r, k]) <= slack + (2 if dtype == "bf16" else 0)
    for e, n, k in [(0, 0, 0), (1, 3, 3), (2, 23, 39), (3, 10, 1)]:
        b = w.clone()
        b[e, n, k] += 1
        assert abs(value(a, b) - value(a, w) - dw[e, n, k]) <= slack * 20 + (2 if dtype == "bf16" else 0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,N,K,pad", [(40, 64, 64, 0), (300, 264, 136, 8), (70, 33, 77, 3)])
def test_infinities_and_nan_stay_where_they_are(kernel, rows, N, K, pad, dtype):
    """Padding of the rows, rows of other experts, rows of none: what is not part of an element's sum does not reach it."""
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(rows)
    counts = [rows // 2, rows - rows // 2 - 3]
    a, w = _normal(gen, rows, K).to(types[dtype]), _normal(gen, 2, N, K).to(types[dtype])
    a[1, K - 1], a[rows // 2, 0] = float("inf"), float("nan")
    w[1, N - 1, 0] = float("nan")
    _, av = _padded(a, pad, float("nan"))
    av[sum(counts):] = float("nan")
    offsets, L = _offsets(counts), _lib()
    c = _np(L.lcma_gemm_experts(av, offsets, w))
    bad = np.zeros((rows, N), bool)
    bad[1], bad[rows // 2] = True, True
    bad[rows // 2:sum(counts), N - 1] = True
    assert np.array_equal(~np.isfinite(c), bad)
    _, dc = _padded(_normal(gen, rows, N).to(types[dtype]), pad, float("nan"))
    dc[sum(counts):] = float("nan")
    dw = _np(L.lcma_gemm_experts_grad(dc, av, offsets))
    bad = np.zeros((2, N, K), bool)
    bad[0, :, K - 1], bad[1, :, 0] = True, True
    assert np.array_equal(~np.isfinite(dw), bad)


def test_offsets_outside_the_rows_reach_nothing():
    """Row numbers are held to the rows there are, and a group that ends before it begins is empty."""
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(1)
    a, w = _whole(gen, 20, 64).bfloat16(), _whole(gen, 3, 72, 64).bfloat16()
    offsets = torch.tensor([0, 5, 3, 1 << 30], dtype=torch.int32, device="cuda")
    c = torch.full((24, 72), 9.0, device="cuda").bfloat16()
    L = _lib()
    L.lcma_gemm_experts(a, offsets, w, c[:20])
    # (rows 3 and 4 are the first expert's and the last one's: either may be there)
    assert np.array_equal(_np(c[5:20]), _rounded(X.gemm_experts(_np(a[5:]), [0, 15], _np(w[2:])), "bf16")) and (c[20:] == 9.0).all()
    assert np.array_equal(_np(c[:3]), _rounded(X.gemm_experts(_np(a[:3]), [0, 3], _np(w[:1])), "bf16"))
    dw = _np(L.lcma_gemm_experts_grad(a, a, offsets))
    assert np.array_equal(dw, _rounded(X.gemm_experts_grad(_np(a), _np(a), [0, 5, 5, 20]) * [[[1]], [[0]], [[1]]] + np.array([0, 0, 1])[:, None, None] *
                                       X.gemm_experts_grad(_np(a), _np(a), [0, 3, 5])[1], "bf16"))


def test_offsets_that_do_not_ascend_write_nothing_else(kernel):
    """What the rows hold then is not specified; what lies around them stays, and other calls are right."""
    torch, types = _torch()
    L, gen = _lib(), torch.Generator(device="cuda").manual_seed(5)
    rows, N, K, E = 300, 136, 72, 64
    a, w = _whole(gen, rows, K).bfloat16(), _whole(gen, E, N, K).bfloat16()
    room = torch.full((rows + 20, N), 7.0, device="cuda").bfloat16()
    weights = torch.full((E + 2, N, K), 7.0, device="cuda").bfloat16()
    for values in ([0, rows] * 32 + [0], [rows, 0] * 32 + [rows], [0, 2 ** 31 - 1] * 32 + [5], [-2 ** 31, 2 ** 31 - 1] * 32 + [7]):
        offsets = torch.tensor(values, dtype=torch.int32, device="cuda")
        L.lcma_gemm_experts(a, offsets, w, room[10:-10])
        L.lcma_gemm_experts_grad(room[10:-10].nan_to_num(0.0), a, offsets, weights[1:-1])
        torch.cuda.synchronize()
        assert all((t == 7.0).all() for t in (room[:10], room[-10:], weights[0], weights[-1]))
    right = L.lcma_gemm_experts(a, torch.tensor([0] * 64 + [rows], dtype=torch.int32, device="cuda"), w)
    assert torch.equal(right, (a.float() @ w[-1].float().t()).bfloat16())


def test_empty_calls():
    torch, types = _torch()
    L, new = _lib(), lambda *s: torch.full(s, 5.0, device="cuda").bfloat16()
    o = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    assert L.lcma_gemm_experts(new(0, 8), o(0, 0), new(1, 16, 8)).shape == (0, 16)
    assert L.lcma_gemm_experts(new(4, 8), o(0, 4), new(1, 0, 8)).shape == (4, 0)
    assert (L.lcma_gemm_experts(new(4, 0), o(0, 3), new(1, 16, 0)) == 0).all()
    assert (L.lcma_gemm_experts_grad(new(0, 16), new(0, 8), o(0, 0, 0)) == 0).all()
    assert L.lcma_gemm_experts_grad(new(3, 0), new(3, 8), o(0, 3)).shape == (1, 0, 8)


@pytest.mark.parametrize("counts,N,K", [([1, 0, 1], 264, 520), ([200, 0, 311], 264, 328), ([40, 70], 77, 33)])
def test_captured_and_replayed(kernel, counts, N, K):
    """New rows, weights and offsets in the same places: every replay gives the eager calls' bits."""
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(9)
    rows, E, L = sum(counts), len(counts), _lib()
    a, w, dc = (_normal(gen, *s).bfloat16() for s in ((rows, K), (E, N, K), (rows, N)))
    offsets = _offsets(counts)
    run = lambda: (L.lcma_gemm_experts(a, offsets, w), L.lcma_gemm_experts(dc, offsets, w, b_nk=False), L.lcma_gemm_experts_grad(dc, a, offsets))
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for i in range(3):
        for t in (a, w, dc):
            t.copy_(_normal(gen, *t.shape))
        offsets.copy_(_offsets(counts[i:] + counts[:i]))
        want = run()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want))


def test_two_streams_at_once_and_repeated_calls_give_the_same_bits():
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(11)
    a, w, dc = (_normal(gen, *s).bfloat16() for s in ((700, 520), (4, 264, 520), (700, 264)))
    offsets, L = _offsets([300, 0, 250, 100]), _lib()
    run = lambda: (L.lcma_gemm_experts(a, offsets, w), L.lcma_gemm_experts(dc, offsets, w, b_nk=False), L.lcma_gemm_experts_grad(dc, a, offsets))
    want = run()
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(run())
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for g in got for x, y in zip(g, want))
