"""4-bit weights with group scales: lcma_i4_quantize, lcma_i4_prepare, lcma_i4_gemm_nt, lcma_i4_gemm_experts against their definitions in 64 bits.

What the products may be off by: inside a group the fp32 terms are x (24 + q) / 16 and -1.5 x, 2 group of them, every addition off by at most 2^-23 of a partial
sum of up to sum |x| (1.94 + 1.5): 2 group 2^-23 3.5 sum |x| 16 S; the sums of the groups, times 16 S, are added in fp32: 2 groups 2^-23 sum |x q S|; then half a step of C's type
(fp32: the scale's product and the bias, 2^-24 each)."""
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


@pytest.fixture(params=["", "16x16", "16x32", "16x64", "64x64"], scope="module")
def kernel(request):
    """The kernel of the rule, and every kernel by name."""
    _lib().lcma_set_tuning("i4_kernel", request.param)
    yield request.param
    _lib().lcma_set_tuning("i4_kernel", "")


def _np(t):
    return t.double().cpu().numpy()


def _weights(gen, lead, N, K, group):
    torch, _ = _torch()
    codes = torch.randint(-8, 8, (*lead, N, K), device="cuda", generator=gen).to(torch.int8)
    scales = torch.rand((*lead, N, -(-K // group)), device="cuda", generator=gen) * 0.02 + 0.001
    return codes, scales


def _close(got, x, q, s, group, bias, dtype):
    torch, types = _torch()
    K = x.shape[1]
    want = x @ X.i4_dequantize(q, s, group).T + bias
    sums = np.abs(x) @ np.repeat(np.abs(s).astype(np.float64), group, axis=1)[:, :K].T
    terms = np.abs(x) @ np.abs(X.i4_dequantize(q, s, group)).T
    step = torch.finfo(types[dtype]).eps / 2
    tolerance = (2 * group * 3.5 * 16 * 2.0 ** -23 * sums + (2 * s.shape[1] * 2.0 ** -23 + 2.0 ** -24) * (terms + np.abs(bias))) * (1 + step) + 2 * step * np.abs(want)
    if dtype != "f32":
        tolerance -= step * np.abs(want)
    assert (np.abs(got - want) <= tolerance).all(), float((np.abs(got - want) - tolerance).max())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K,pad,bias", [(1, 1, 1, 0, False), (1, 64, 128, 0, True), (1, 272, 4096, 0, False), (3, 33, 77, 3, True), (16, 48, 2200, 8, False), (17, 200, 520, 0, True),
                                            (45, 101, 1545, 24, True), (64, 128, 256, 0, False), (100, 130, 300, 5, False), (257, 144, 1100, 0, True)])
def test_linear(kernel, M, N, K, pad, bias, group, dtype):
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(M + N + K)
    codes, scales = _weights(gen, (), N, K, group)
    xw = torch.full((M, K + pad), float("nan"), device="cuda").to(types[dtype])
    x = xw[:, :K]
    x.copy_(torch.randn((M, K), device="cuda", generator=gen))
    b = torch.randn((N,), device="cuda", generator=gen) if bias else None
    cw = torch.full((M + 1, N + pad), 7.0, device="cuda").to(types[dtype])
    L = _lib()
    wp = L.lcma_i4_prepare(codes, scales, group)
    assert wp.numel() == L.lcma_i4_prepared_bytes(N, K, group)
    c = L.lcma_i4_gemm_nt(x, wp, cw[:M, :N], group, b)
    _close(_np(c), _np(x), _np(codes), _np(scales), group, _np(b) if bias else 0.0, dtype)
    assert (cw[:, N:] == 7.0).all() and (cw[M:] == 7.0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("counts,behind,N,K,group,bias", [([1, 0, 1], 0, 264, 520, 128, False), ([0, 5, 2, 0, 16], 3, 77, 300, 32, True), ([17, 40, 0, 3], 0, 130, 1100, 64, False),
                                                          ([1] * 70, 5, 40, 136, 128, True), ([100, 33], 1, 200, 260, 64, True), ([0, 0], 4, 24, 64, 32, True)], ids=str)
def test_experts(kernel, counts, behind, N, K, group, bias, dtype):
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(N + K)
    E, n = len(counts), sum(counts)
    codes, scales = _weights(gen, (E,), N, K, group)
    x = torch.randn((n + behind, K), device="cuda", generator=gen).to(types[dtype])
    x[n:] = float("nan")
    b = torch.randn((E, N), device="cuda", generator=gen) if bias else None
    offsets = torch.tensor(np.cumsum([0] + counts), dtype=torch.int32, device="cuda")
    L = _lib()
    c = torch.full((n + behind, N), 9.0, device="cuda").to(types[dtype])
    L.lcma_i4_gemm_experts(x, offsets, L.lcma_i4_prepare(codes, scales, group), c, group, b)
    at = np.cumsum([0] + counts)
    for e in range(E):
        if counts[e]:
            _close(_np(c[at[e]:at[e + 1]]), _np(x[at[e]:at[e + 1]]), _np(codes[e]), _np(scales[e]), group, _np(b[e]) if bias else 0.0, dtype)
    assert (c[n:] == 0).all()


@pytest.mark.parametrize("group", [32, 64, 128])
def test_every_code_in_every_place(kernel, group):
    """One row of X with a single one at a time: C is the column of weights, exactly (16 S q / 16 in fp32, scales are powers of two)."""
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(group)
    N, K = 48, 300
    codes = torch.randint(-8, 8, (N, K), device="cuda", generator=gen).to(torch.int8)
    scales = torch.exp2(torch.randint(-6, 6, (N, -(-K // group)), device="cuda", generator=gen).float())
    L = _lib()
    c = L.lcma_i4_gemm_nt(torch.eye(K, device="cuda"), L.lcma_i4_prepare(codes, scales, group), torch.empty((K, N), device="cuda"), group)
    assert np.array_equal(_np(c).T, X.i4_dequantize(_np(codes), _np(scales), group))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("experts,N,K,pad", [(0, 1, 1, 0), (0, 50, 300, 0), (3, 17, 129, 3), (2, 64, 256, 8)])
def test_quantised_weights(experts, N, K, pad, group, dtype):
    """The codes and scales of the definition, bit for bit: what the library lays out equals what lcma_i4_prepare lays out of them."""
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(N)
    lead = (experts,) if experts else ()
    w = torch.randn((*lead, N, K + pad), device="cuda", generator=gen).to(types[dtype])[..., :K]
    flat = _np(w).reshape(-1, K)
    flat[0, : min(K, 40)] = 0
    if flat.shape[0] > 5 and K > 200:
        flat[1, 3], flat[2, 199], flat[3] = np.inf, np.nan, 1e-39 if dtype == "f32" else 2.0 ** -14
    w.copy_(torch.from_numpy(flat).reshape(w.shape))
    L = _lib()
    got = L.lcma_i4_quantize(w, group)
    q, s = X.i4_quantize(flat, group)
    put = lambda v: torch.from_numpy(v).cuda().reshape(*lead, N, -1)
    want = L.lcma_i4_prepare(put(q), put(s), group)
    assert got.shape == (*lead, L.lcma_i4_prepared_bytes(N, K, group))
    same = (got == want).cpu().numpy()
    if not same.all():  # (NaN scales may differ in their bits)
        a, b = got.cpu().numpy().reshape(-1, 4).view(np.float32), want.cpu().numpy().reshape(-1, 4).view(np.float32)
        off = ~same.reshape(-1, 4).all(axis=1)
        assert np.isnan(a[off]).all() and np.isnan(b[off]).all()


def test_a_quantised_layer_is_near_the_unquantised_one():
    """A code is off by at most half of S, S = max / 7 of a group: for normal weights and 128 to a group (max about 2.6) 0.107 rms of a weight's spread, and so of the result."""
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(8)
    x, w = (torch.randn(s, device="cuda", generator=gen).bfloat16() for s in ((40, 1024), (256, 1024)))
    L = _lib()
    c = _np(L.lcma_i4_gemm_nt(x, L.lcma_i4_quantize(w), torch.empty((40, 256), device="cuda").bfloat16()))
    want = _np(x) @ _np(w).T
    assert 0.05 <= np.linalg.norm(c - want) / np.linalg.norm(want) <= 0.16


def test_infinities_and_nan_stay_in_their_rows():
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(4)
    for M in (5, 40):
        codes, scales = _weights(gen, (), 40, 200, 64)
        scales[7, 1] = float("nan")
        x = torch.randn((M, 200), device="cuda", generator=gen).bfloat16()
        x[1, 199], x[M - 1, 0] = float("inf"), float("nan")
        L = _lib()
        c = _np(L.lcma_i4_gemm_nt(x, L.lcma_i4_prepare(codes, scales, 64), torch.empty((M, 40), device="cuda").bfloat16(), 64))
        bad = np.zeros((M, 40), bool)
        bad[1], bad[M - 1], bad[:, 7] = True, True, True
        assert np.array_equal(~np.isfinite(c), bad)


def test_empty_calls():
    torch, types = _torch()
    L, e = _lib(), lambda *s, t="bfloat16": torch.empty(s, device="cuda", dtype=getattr(torch, t))
    wp = L.lcma_i4_prepare(e(16, 0, t="int8"), e(16, 0, t="float32"))
    assert wp.numel() == 0
    bias = torch.arange(16.0, device="cuda")
    assert torch.equal(L.lcma_i4_gemm_nt(e(3, 0), wp, e(3, 16), 128, bias).float(), bias.expand(3, 16))
    assert (L.lcma_i4_gemm_nt(e(3, 0), wp, e(3, 16)) == 0).all()
    wp = L.lcma_i4_quantize(e(0, 64))
    assert L.lcma_i4_gemm_nt(e(3, 64), wp, e(3, 0)).shape == (3, 0) and L.lcma_i4_gemm_nt(e(0, 64), wp, e(0, 0)).shape == (0, 0)


@pytest.mark.parametrize("M", [1, 30])
def test_captured_and_replayed(kernel, M):
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(2)
    L = _lib()
    w, x = torch.randn((3, 130, 700), device="cuda", generator=gen).bfloat16(), torch.randn((M, 700), device="cuda", generator=gen).bfloat16()
    offsets = torch.tensor([0, 0, M, M], dtype=torch.int32, device="cuda")
    c, d = (torch.empty((M, 130), device="cuda").bfloat16() for _ in range(2))
    wp = L.lcma_i4_quantize(w)
    run = lambda: (L.lcma_i4_gemm_experts(x, offsets, wp, c), L.lcma_i4_gemm_nt(x, wp[1], d))
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        x.normal_(generator=gen)
        want = [t.clone() for t in run()]
        c.zero_(), d.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c, want[0]) and torch.equal(d, want[1])  # (c and d may be two kernels', whose sums are cut elsewhere)
