"""The 8-bit-integer linear layer, alone and over experts, against the plain forms of oracle/experts.py: codes and scales bit for bit (the
gated ones within what the fp32 gate may be off), products within the rounding of their scaling and of C."""
import numpy as np
import pytest

import lcma_inputs as inp
from oracle import experts as X

pytestmark = pytest.mark.gpu

HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # of the storage types, relative
ES = {"f32": 4, "bf16": 2, "f16": 2}


def _values(rng, shape, dt, spread=1.0):
    """Stored values and the same as float64."""
    stored = inp.store(rng.standard_normal(shape) * spread, dt)
    return stored, inp.widen(stored, dt).astype(np.float64)


def _codes(rng, lead, rows, K):
    """Random codes on the device, rows padded with zeros to the code pitch, and the same without padding."""
    import torch
    q = rng.integers(-127, 128, (*lead, rows, K)).astype(np.int8)
    padded = np.zeros((*lead, rows, (K + 127) // 128 * 128), np.int8)
    padded[..., :K] = q
    return torch.from_numpy(padded).cuda(), q


def _strided(rows, cols, dt, pad, fill):
    """A rows x cols view into a larger tensor of `fill`: `pad` unused columns in front and behind, an unused row on either side."""
    import torch
    td = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dt]
    whole = torch.full((rows + 2, cols + 2 * pad), fill, dtype=td, device="cuda")
    return whole, whole[1:1 + rows, pad:pad + cols]


def _untouched(whole, rows, cols, pad):
    import torch
    outside = torch.ones(whole.shape, dtype=torch.bool, device="cuda")
    outside[1:1 + rows, pad:pad + cols] = False
    return torch.isnan(whole[outside]).all().item()


def _host(t, dt):
    import gpu_util as G
    return G.to_host_f64(t, dt).astype(np.float64)


def _device(stored, dt):
    import gpu_util as G
    return G.to_device(stored, dt)


# ------------------------------------------------------------------ quantisation
@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,K,pad", [(1, 1, 0), (3, 7, 1), (5, 8, 0), (2, 127, 0), (4, 128, 0), (3, 129, 3), (7, 1000, 0), (2, 2047, 5), (3, 2048, 8),
                                        (2, 2049, 0), (300, 72, 0), (2, 14336, 0), (1, 20001, 1), (2, 40000, 0)])
def test_codes_and_scales(dt, rows, K, pad):
    import torch
    from paper_2605_06057_amd import binding as B
    rng = np.random.default_rng(rows * 100003 + K)
    stored, x = _values(rng, (rows, K), dt, 3.0)
    whole, view = _strided(rows, K, dt, pad, float("nan"))
    view.copy_(_device(stored, dt))
    pitch = B.lcma_i8_code_pitch(K)
    Q = torch.full((rows + 1, pitch), 99, dtype=torch.int8, device="cuda")
    S = torch.full((rows + 1,), float("nan"), device="cuda")
    B.lcma_i8_quantize(view, Q[:rows], S[:rows])
    torch.cuda.synchronize()
    q, s = X.i8_quantize(x)
    assert np.array_equal(S[:rows].cpu().numpy(), s) and torch.isnan(S[rows]).item()
    got = Q.cpu().numpy()
    assert np.array_equal(got[:rows, :K], q) and (got[:rows, K:] == 0).all() and (got[rows] == 99).all()


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
def test_rows_that_are_hard_to_scale(dt):
    """Zeros, one value alone, subnormals, the largest values, ties, infinities and NaN in one row of many."""
    import torch
    from paper_2605_06057_amd import binding as B
    K = 1000
    rng = np.random.default_rng(5)
    x = rng.standard_normal((12, K))
    x[0] = 0
    x[1] = 0
    x[1, 777] = -2.5
    x[2] *= 2.0 ** (-140 if dt != "f16" else -22)                       # subnormal in fp32 and bf16 (fp16: its own)
    x[3] = rng.choice([-1.0, 1.0], K) * {"f32": 3.4028234663852886e38, "bf16": 3.3895313892515355e38, "f16": 65504.0}[dt]
    x[4] = rng.integers(-254, 255, K) / 2.0                             # amax 127: every half is a tie
    x[4, 0] = 127
    x[5, 3] = np.inf
    x[6, 999] = -np.inf
    x[7, 500] = np.nan
    x[8, [1, 2]] = np.inf, np.nan
    x[9] = -0.0
    x[10] *= 2.0 ** -101 if dt != "f16" else 1.0
    stored = inp.store(x, dt)
    Q, S = B.lcma_i8_quantize(_device(stored, dt))
    q, s = X.i8_quantize(inp.widen(stored, dt).astype(np.float64))
    assert np.array_equal(Q.cpu().numpy()[:, :K], q)
    got = S.cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(s)) and np.array_equal(got[~np.isnan(s)], s[~np.isnan(s)])
    # and what becomes of such rows in a product: NaN for the whole row, zeros for a row of zeros, nothing in other rows
    Wq, w = _codes(rng, (), 65, K)
    Wq[:, 0] = 1
    c = B.lcma_i8_gemm_nt(Q, S, Wq, torch.ones((65,), device="cuda"), torch.empty((12, 65), device="cuda"), K)
    bad = np.isnan(s) | np.isinf(s)
    host = c.cpu().numpy()
    fine = ~bad & (np.arange(12) != 3)  # (the largest values times a row of weights are past the range of fp32)
    assert np.isnan(host[bad]).all() and np.isfinite(host[fine]).all() and (host[[0, 9]] == 0).all()


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,K", [(1, 1), (3, 77), (2, 128), (5, 1001), (2, 2056), (2, 14336), (1, 17000)])
def test_gated(dt, rows, K):
    """The gate is formed in fp32 with the fast exponential and division, off by at most 2^-18 of the value for |g| up to 90 (2^-22 |g| from the
    argument of the exponential, some units in the last place from the rest); so is the scale, and a code is the rounded quotient of two such."""
    import torch
    from paper_2605_06057_amd import binding as B
    rng = np.random.default_rng(K)
    stored, x = _values(rng, (rows, 2 * K), dt, 2.0)
    Q, S = B.lcma_i8_quantize(_device(stored, dt), gated=True)
    v = X.silu_gate(x)
    amax, off = np.abs(v).max(axis=1), 2.0 ** -18
    s, q = S.cpu().numpy().astype(np.float64), Q.cpu().numpy()
    assert np.all(np.abs(s - amax / 127) <= amax / 127 * off) and (q[:, K:] == 0).all()
    assert np.all(np.abs(q[:, :K] - v / (amax[:, None] / 127)) <= 0.5 + 127 * 2 * off)
    assert (np.abs(q).max(axis=1) == 127).all()


def test_gate_at_the_ends():
    """Gates whose exponential overflows, and infinities."""
    import torch
    from paper_2605_06057_amd import binding as B
    x = torch.tensor([[-200.0, 1.0, 2.0, 3.0], [-1e38, 0.0, 1.0, 5.0], [200.0, 1.0, 1.0, 1.0], [float("inf"), 1.0, 1.0, 1.0], [float("-inf"), 1.0, 1.0, 1.0]],
                     device="cuda")
    Q, S = B.lcma_i8_quantize(x, gated=True)
    q, s = Q.cpu().numpy()[:, :2], S.cpu().numpy()
    assert q[0].tolist() == [0, 127] and abs(s[0] * 127 - 3 / (1 + np.exp(-1.0))) < 1e-5
    assert q[1].tolist() == [0, 0] and s[1] == 0
    assert q[2].tolist() == [127, 0] and abs(s[2] * 127 - 200) < 1e-3
    assert np.isinf(s[3]) and np.isnan(s[4])


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("gate", [-80.0, -86.0, -88.0, -89.0, -92.0, -100.0, -150.0, -170.0])
def test_gates_far_below_zero(dt, gate):
    """silu(g) there is |g| exp(g), a small number and not zero, up to where exp(-g) has left fp32 (88.7) and beyond: rows in which all gates are of that size, times
    large linear parts.  The gate is off by at most 2^-18 of the value (test_gated); below 2^-126 a value has an error of 2^-149 besides."""
    from paper_2605_06057_amd import binding as B
    rng = np.random.default_rng(int(-gate))
    K, up = 777, {"f32": 2.0 ** 120, "bf16": 2.0 ** 120, "f16": 2.0 ** 14}[dt]
    stored = inp.store(np.concatenate([gate + rng.uniform(-2, 2, (3, K)), rng.uniform(-3, 3, (3, K)) * up], axis=1), dt)
    v = X.silu_gate(inp.widen(stored, dt).astype(np.float64))
    if np.abs(v).max(axis=1).min() < 2.0 ** -120:
        return  # (fp16: nothing that fp32 can tell from zero)
    Q, S = B.lcma_i8_quantize(_device(stored, dt), gated=True)
    s, q, amax, off = S.cpu().numpy().astype(np.float64), Q.cpu().numpy(), np.abs(v).max(axis=1), 2.0 ** -18
    assert np.all(np.abs(s - amax / 127) <= amax / 127 * off + 2.0 ** -149)
    room = 0.5 + 127 * 2 * off + 2.0 ** -148 / (amax / 127)
    assert np.all(np.abs(q[:, :K] - v / (amax[:, None] / 127)) <= room[:, None]) and (np.abs(q).max(axis=1) == 127).all()


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tokens,top_k,K", [(1, 1, 1), (5, 2, 129), (33, 8, 520), (70, 3, 2051)])
def test_quantised_while_dispatching(dt, tokens, top_k, K):
    import torch
    from paper_2605_06057_amd import binding as B
    rng = np.random.default_rng(tokens + K)
    stored, x = _values(rng, (tokens, K), dt)
    ids = torch.from_numpy(rng.integers(-1, 6, (tokens, top_k)).astype(np.int32)).cuda()
    order, position, offsets = B.lcma_tokens_sort(ids, 6)
    n, pitch = tokens * top_k, B.lcma_i8_code_pitch(K)
    Q, S = torch.full((n, pitch), 99, dtype=torch.int8, device="cuda"), torch.full((n,), -1.0, device="cuda")
    B.lcma_i8_quantize_dispatch(_device(stored, dt), position, Q, S)
    q, s = X.i8_quantize(x)
    token, kept = order.cpu().numpy() // top_k, int(offsets[-1])
    Q, S = Q.cpu().numpy(), S.cpu().numpy()
    assert np.array_equal(Q[:kept, :K], q[token[:kept]]) and (Q[:kept, K:] == 0).all() and np.array_equal(S[:kept], s[token[:kept]])
    assert (Q[kept:] == 99).all() and (S[kept:] == -1).all()


# ------------------------------------------------------------------ products
def _check(got, want, dt, bias):
    """The sum is turned into fp32, scaled twice and, with a bias, added to it: 2^-24 of the value each; then the rounding of C."""
    room = np.abs(want - (0 if bias is None else bias)) * 3.1 * 2.0 ** -24 + np.abs(want) * (1.01 * 2.0 ** -24 + 1.001 * HALF_ULP[dt]) + 2.0 ** -25
    worst = np.max(np.abs(got - want) - room)
    assert worst <= 0, f"{worst:.3e} more than the roundings allow"


SHAPES = [(1, 1, 1), (1, 14336, 256), (2, 17, 127), (1, 4096, 4096), (15, 33, 128), (16, 16, 129), (17, 65, 640), (31, 1000, 1000), (33, 127, 2176), (45, 1001, 1545),
          (63, 4099, 384), (64, 64, 128), (65, 128, 512), (128, 257, 4224), (129, 255, 130), (200, 2048, 1024), (255, 513, 256), (256, 256, 896), (257, 1025, 384),
          (600, 770, 1153), (1025, 1536, 640), (2049, 2304, 257), (4100, 72, 1000), (70, 8200, 300)]


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("M,N,K", SHAPES, ids=lambda v: str(v))
def test_product(dt, M, N, K):
    import torch
    from paper_2605_06057_amd import binding as B
    rng = np.random.default_rng(M + 7 * N + 31 * K)
    Aq, a = _codes(rng, (), M, K)
    Wq, w = _codes(rng, (), N, K)
    sa, sw = (rng.uniform(0.5, 1.5, M) / 127).astype(np.float32), (rng.uniform(0.5, 1.5, N) / 127).astype(np.float32)
    dev = lambda v: torch.from_numpy(v).cuda()
    for pad, bias in ((0, None), (1, rng.standard_normal(N).astype(np.float32)), (4, None)):
        whole, c = _strided(M, N, dt, pad, float("nan"))
        print(f"product {dt} {M}x{N}x{K} pad {pad}", flush=True)
        B.lcma_i8_gemm_nt(Aq, dev(sa), Wq, dev(sw), c, K, None if bias is None else dev(bias))
        torch.cuda.synchronize()
        _check(_host(c, dt), X.i8_gemm(a, sa, w, sw, bias), dt, bias)
        assert _untouched(whole, M, N, pad), "wrote outside C"


def test_largest_sums_are_exact():
    """K at its limit with codes of -128 and 127 in every place: sums up to 2^31 - 2^14 do not wrap."""
    import torch
    from paper_2605_06057_amd import binding as B
    K = 131071
    pitch = B.lcma_i8_code_pitch(K)
    Aq, Wq = torch.zeros((3, pitch), dtype=torch.int8, device="cuda"), torch.zeros((5, pitch), dtype=torch.int8, device="cuda")
    Aq[0, :K], Aq[1, :K], Aq[2, :K] = -128, 127, 1
    Wq[0, :K], Wq[1, :K], Wq[2, :K], Wq[3, :K:2], Wq[4, K - 1] = -128, 127, 1, 1, 1
    one = torch.ones((5,), device="cuda")
    c = B.lcma_i8_gemm_nt(Aq, one[:3], Wq, one, torch.empty((3, 5), device="cuda"), K).cpu().double()
    want = (Aq.cpu().double() @ Wq.cpu().double().t()).float().double()
    assert torch.equal(c, want)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_empty_k_gives_the_bias(dt):
    import torch
    from paper_2605_06057_amd import binding as B
    x = torch.empty((5, 0), device="cuda")
    Q, S = B.lcma_i8_quantize(x)
    assert Q.shape == (5, 0) and (S == 0).all().item()
    Wq, sw, bias = torch.empty((70, 0), dtype=torch.int8, device="cuda"), torch.ones((70,), device="cuda"), torch.arange(70.0, device="cuda")
    td = {"f32": torch.float32, "bf16": torch.bfloat16}[dt]
    for b in (bias, None):
        c = B.lcma_i8_gemm_nt(Q, S, Wq, sw, torch.full((5, 70), float("nan"), device="cuda", dtype=td), 0, b)
        assert torch.equal(c.float(), (bias if b is not None else 0 * bias).expand(5, 70))


COUNTS = [[1], [0, 1, 0], [3, 0, 5, 1], [64, 64, 1], [65, 0, 0, 200, 7, 0, 31], [1] * 8 + [0] * 8, [0] * 7 + [300], [16, 17, 32, 33, 48, 100, 128, 129], [2] * 130, [0] * 100 + [5] + [0] * 99 + [70]]


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("counts,behind", [(c, b) for c in COUNTS for b in (0, 5)] + [([0, 0, 0], 9), ([256, 255, 300, 1, 700], 300)],
                         ids=lambda v: str(v).replace(" ", "")[:30])
def test_experts(dt, counts, behind):
    import torch
    from paper_2605_06057_amd import binding as B
    E, rows = len(counts), sum(counts) + behind
    N, K = (136, 200) if E > 20 else (515, 1000)
    rng = np.random.default_rng(rows + E)
    Aq, a = _codes(rng, (), rows, K)
    Wq, w = _codes(rng, (E,), N, K)
    sa, sw = (rng.uniform(0.5, 1.5, rows) / 127).astype(np.float32), (rng.uniform(0.5, 1.5, (E, N)) / 127).astype(np.float32)
    sa[sum(counts):] = np.nan  # rows behind the experts' are not read
    offsets = np.cumsum([0] + counts).astype(np.int32)
    dev = lambda v: torch.from_numpy(v).cuda()
    for pad, bias in ((0, None), (3, rng.standard_normal((E, N)).astype(np.float32))):
        whole, c = _strided(rows, N, dt, pad, float("nan"))
        print(f"experts {dt} {counts} {behind} pad {pad}"[:200], flush=True)
        B.lcma_i8_gemm_experts(Aq, dev(sa), dev(offsets), Wq, dev(sw), c, K, None if bias is None else dev(bias))
        torch.cuda.synchronize()
        sa0 = np.where(np.isnan(sa), 0, sa)
        want = X.i8_gemm_experts(a, sa0, offsets, w, sw, bias)
        row_bias = None if bias is None else np.concatenate([np.repeat(bias.astype(np.float64), counts, axis=0), np.zeros((behind, N))])
        _check(_host(c, dt), want, dt, row_bias)
        assert _untouched(whole, rows, N, pad), "wrote outside C"


@pytest.mark.parametrize("per,E,N,K", [(1, 8, 4096, 1024), (3, 8, 2048, 1000), (20, 16, 1500, 512), (90, 60, 1408, 384), (300, 8, 1024, 640), (1100, 4, 1030, 384)])
def test_experts_of_many_sizes(per, E, N, K):
    """About `per` rows for each expert (none for some), every column and row compared exactly: integers up to 2^24 in fp32."""
    import torch
    from paper_2605_06057_amd import binding as B
    rng = np.random.default_rng(per + E)
    counts = rng.integers(0, 2 * per + 1, E)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    rows = int(offsets[-1])
    gen = torch.Generator(device="cuda").manual_seed(per)
    pitch = B.lcma_i8_code_pitch(K)
    Aq, Wq = torch.zeros((rows, pitch), dtype=torch.int8, device="cuda"), torch.zeros((E, N, pitch), dtype=torch.int8, device="cuda")
    Aq[:, :K] = torch.randint(-100, 101, (rows, K), device="cuda", generator=gen)
    Wq[:, :, :K] = torch.randint(-100, 101, (E, N, K), device="cuda", generator=gen)
    c = torch.full((rows, N), float("nan"), device="cuda")
    B.lcma_i8_gemm_experts(Aq, torch.ones((rows,), device="cuda"), torch.from_numpy(offsets).cuda(), Wq, torch.ones((E, N), device="cuda"), c, K)
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        assert torch.equal(c[a:b], Aq[a:b].float() @ Wq[e].float().t())


def test_weights_that_pass_32_bits():
    """Experts whose codes lie further than 4 GiB from the first one's, and rows of C further than 4 GiB from its first."""
    import torch
    from paper_2605_06057_amd import binding as B
    E, N, K = 5, 65536, 16384
    Wq = torch.zeros((E, N, K), dtype=torch.int8, device="cuda")
    Wq[4, 65500:] = 3
    Wq[4, :, 16000:] = 2
    offsets = torch.tensor([0, 1, 1, 1, 1, 6], dtype=torch.int32, device="cuda")
    Aq = torch.ones((6, K), dtype=torch.int8, device="cuda")
    whole = torch.empty((6, 400_000_000), dtype=torch.bfloat16, device="cuda")
    c = whole[:, :N]
    B.lcma_i8_gemm_experts(Aq, torch.ones((6,), device="cuda"), offsets, Wq, torch.ones((E, N), device="cuda"), c, K)
    want = torch.full((N,), 2.0 * 384, device="cuda")
    want[65500:] = 3 * 16000 + 2 * 384
    assert (c[0] == 0).all().item() and (c[1:] == want.bfloat16()).all().item()


KERNELS = ["16x16", "32x32", "64x64", "64x128", "128x128", "128x256", "256x256"]


@pytest.fixture
def kernel(request):
    from paper_2605_06057_amd import binding as B
    B.lcma_set_tuning("i8_kernel", request.param)
    yield request.param
    B.lcma_set_tuning("i8_kernel", "")


@pytest.mark.parametrize("kernel", KERNELS, indirect=True)
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (17, 65, 128), (64, 256, 257), (129, 255, 130), (300, 520, 1000), (257, 1025, 384), (1025, 1536, 640)], ids=lambda v: str(v))
def test_product_on_every_kernel(kernel, M, N, K):
    for dt in ("f32", "bf16", "f16"):
        test_product(dt, M, N, K)


@pytest.mark.parametrize("kernel", KERNELS, indirect=True)
@pytest.mark.parametrize("counts,behind", [([3, 0, 5, 1], 2), ([65, 0, 0, 200, 7, 0, 31], 0), ([2] * 130, 1), ([256, 255, 300, 1, 700], 300)], ids=lambda v: str(v).replace(" ", "")[:30])
def test_experts_on_every_kernel(kernel, counts, behind):
    test_experts("bf16", counts, behind)


def test_an_unknown_kernel_is_the_default():
    from paper_2605_06057_amd import binding as B
    B.lcma_set_tuning("i8_kernel", "7x9")
    try:
        test_product("bf16", 33, 127, 256)
    finally:
        B.lcma_set_tuning("i8_kernel", "")


def test_many_rows():
    """More rows than a grid has in its second dimension, quantised and multiplied; sums below 2^24 are exact in fp32."""
    import torch
    from paper_2605_06057_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(8)
    M, N, K = 70001, 40, 72
    x = torch.randint(-127, 128, (M, K), device="cuda", generator=gen).float()
    x[:, 0] = 127  # scale 1: the codes are the values
    Q, S = B.lcma_i8_quantize(x)
    assert torch.equal(Q[:, :K].float(), x) and (Q[:, K:] == 0).all().item() and (S == 1).all().item()
    Wq = torch.zeros((N, 128), dtype=torch.int8, device="cuda")
    Wq[:, :K] = torch.randint(-127, 128, (N, K), device="cuda", generator=gen)
    c = B.lcma_i8_gemm_nt(Q, S, Wq, torch.ones((N,), device="cuda"), torch.empty((M, N), device="cuda"), K)
    assert torch.equal(c.double(), x.double() @ Wq[:, :K].double().t())


def test_nothing_to_multiply():
    import torch
    from paper_2605_06057_amd import binding as B
    q, s = B.lcma_i8_quantize(torch.empty((0, 30), device="cuda"))
    w, sw = torch.ones((5, 128), dtype=torch.int8, device="cuda"), torch.ones((5,), device="cuda")
    assert B.lcma_i8_gemm_nt(q, s, w, sw, torch.empty((0, 5), device="cuda"), 30).shape == (0, 5)
    zeros = torch.zeros((3,), dtype=torch.int32, device="cuda")  # no rows for either of two experts
    c = B.lcma_i8_gemm_experts(w[:4], sw[:4], zeros, w.expand(2, 5, 128).contiguous(), sw.expand(2, 5).contiguous(), torch.full((4, 5), float("nan"), device="cuda"), 128)
    assert (c == 0).all().item()


@pytest.mark.parametrize("K", [100, 5000])
def test_quantised_to_rows_that_are_not_there(K):
    """A position of the row behind the last one is left out, as a negative one."""
    import torch
    from paper_2605_06057_amd import binding as B
    rng = np.random.default_rng(K)
    stored, x = _values(rng, (3, K), "bf16")
    n, pitch = 6, B.lcma_i8_code_pitch(K)
    Q, S = torch.full((n + 1, pitch), 99, dtype=torch.int8, device="cuda"), torch.full((n + 1,), -1.0, device="cuda")
    B.lcma_i8_quantize_dispatch(_device(stored, "bf16"), torch.tensor([[4, n], [0, 1], [-1 - n, 5]], dtype=torch.int32, device="cuda"), Q[:n], S[:n])
    q, s = X.i8_quantize(x)
    Q, S = Q.cpu().numpy(), S.cpu().numpy()
    written, token = [4, 0, 1, 5], [0, 1, 1, 2]
    assert np.array_equal(Q[written, :K], q[token]) and (Q[written, K:] == 0).all() and np.array_equal(S[written], s[token])
    assert (Q[[2, 3, n]] == 99).all() and (S[[2, 3, n]] == -1).all()


# ------------------------------------------------------------------ work-groups that walk through several tiles
def _whole_numbers(gen, *shape):
    """Codes of -100 .. 100 on the device, rows padded with zeros to the code pitch."""
    import torch
    out = torch.zeros((*shape[:-1], (shape[-1] + 127) // 128 * 128), dtype=torch.int8, device="cuda")
    out[..., :shape[-1]] = torch.randint(-100, 101, shape, device="cuda", generator=gen)
    return out


WALKS = [(tiles, K) for tiles in (256 + 40, 256 + 200, 512 + 40, 512 + 200) for K in (100, 256, 384, 500, 640, 768)]


@pytest.mark.parametrize("kernel", ["128x256", "256x256"], indirect=True)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("tiles,K", WALKS)
def test_product_of_more_tiles_than_work_groups(kernel, dt, tiles, K):
    """256 work-groups walk through the tiles: a second and a third one, a last round that at most half of them have a tile in and one that more have, 1 to 6
    steps of K, the last tiles along M and N not full.  Whole numbers: sums below 2^24 are exact in fp32, and a rounding to bf16 is the same one."""
    import torch
    from paper_2605_06057_amd import binding as B
    rows, cols = map(int, kernel.split("x"))
    gen = torch.Generator(device="cuda").manual_seed(tiles + K)
    M, N = tiles // 8 * rows - 37, 8 * cols - 61
    Aq, Wq = _whole_numbers(gen, M, K), _whole_numbers(gen, N, K)
    whole, c = _strided(M, N, dt, 3, float("nan"))
    B.lcma_i8_gemm_nt(Aq, torch.ones((M,), device="cuda"), Wq, torch.ones((N,), device="cuda"), c, K)
    assert torch.equal(c, (Aq.float() @ Wq.float().t()).to(c.dtype)) and _untouched(whole, M, N, 3)


@pytest.mark.parametrize("kernel", ["128x256", "256x256"], indirect=True)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("counts", [[130, 0, 4000, 1, 2200, 255, 257, 2500], [5000, 17, 5003, 0, 0, 6000, 300, 129]], ids=["more than 256", "more than 512"])
@pytest.mark.parametrize("K", [100, 256, 384, 500, 640])
def test_experts_of_more_tiles_than_work_groups(kernel, dt, counts, K):
    """The same with groups that end inside tiles and rows behind them."""
    import torch
    from paper_2605_06057_amd import binding as B
    cols, behind, E = int(kernel.split("x")[1]), 301, len(counts)
    gen = torch.Generator(device="cuda").manual_seed(len(counts) + K)
    rows, N = sum(counts) + behind, 8 * cols - 61
    ends = np.cumsum([0] + counts).astype(np.int32)
    Aq, Wq, bias = _whole_numbers(gen, rows, K), _whole_numbers(gen, E, N, K), torch.randint(-50, 51, (E, N), device="cuda", generator=gen).float()
    whole, c = _strided(rows, N, dt, 3, float("nan"))
    one = torch.ones((rows + E * N,), device="cuda")
    B.lcma_i8_gemm_experts(Aq, one[:rows], torch.from_numpy(ends).cuda(), Wq, one[rows:].view(E, N), c, K, bias)
    for e in range(E):
        a, b = int(ends[e]), int(ends[e + 1])
        assert torch.equal(c[a:b], (Aq[a:b].float() @ Wq[e].float().t() + bias[e]).to(c.dtype)), f"expert {e}"
    assert (c[ends[-1]:] == 0).all().item() and _untouched(whole, rows, N, 3)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(8192, 14336, 640), (8191, 14335, 777), (2048, 4096, 1000)])
def test_large_product_by_the_rule(dt, M, N, K):
    import torch
    from paper_2605_06057_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(M + K)
    Aq, Wq = _whole_numbers(gen, M, K), _whole_numbers(gen, N, K)
    c = torch.full((M, N), float("nan"), device="cuda", dtype={"f32": torch.float32, "bf16": torch.bfloat16}[dt])
    B.lcma_i8_gemm_nt(Aq, torch.ones((M,), device="cuda"), Wq, torch.ones((N,), device="cuda"), c, K)
    assert torch.equal(c, (Aq.float() @ Wq.float().t()).to(c.dtype))


# ------------------------------------------------------------------ more rows than some kernel's launch holds
@pytest.mark.parametrize("K", [8, 0])
def test_product_of_very_many_rows(K):
    """2^28 rows: more tiles of 64 x 64 than a launch holds."""
    import torch
    from paper_2605_06057_amd import binding as B
    M, N = (1 << 28) + 5, 3
    Aq, sa = torch.zeros((M, 128 if K else 0), dtype=torch.int8, device="cuda"), torch.ones((M,), device="cuda")
    Wq, bias = torch.zeros((N, 128 if K else 0), dtype=torch.int8, device="cuda"), torch.tensor([0.0, 1.0, 2.0], device="cuda")
    number = torch.arange(M, device="cuda", dtype=torch.int32) % 101
    if K:
        Aq[:, K - 1] = number
        Wq[:, K - 1] = 1
    c = torch.full((M, N), float("nan"), device="cuda", dtype=torch.bfloat16)
    B.lcma_i8_gemm_nt(Aq, sa, Wq, torch.ones((N,), device="cuda"), c, K, bias)
    for n in range(N):
        assert ((c[:, n] == number + n) if K else (c[:, n] == n)).all().item()


def test_the_last_row_number():
    """2^31 - 1 rows (of nothing: K = 0), whose tiles and rows behind the groups end at the last number that 32 bits hold."""
    import torch
    from paper_2605_06057_amd import binding as B
    M = (1 << 31) - 1
    Aq, sa, one = torch.empty((M, 0), dtype=torch.int8, device="cuda"), torch.zeros((M,), device="cuda"), torch.ones((2, 1), device="cuda")
    Wq, bias = torch.empty((2, 1, 0), dtype=torch.int8, device="cuda"), torch.tensor([[3.0], [5.0]], device="cuda")
    c = torch.full((M, 1), float("nan"), device="cuda", dtype=torch.bfloat16)
    B.lcma_i8_gemm_nt(Aq, sa, Wq[0], one[0], c, 0, bias[0])
    assert (c == 3).all().item()
    for offsets in ([0, 7, 1000], [0, 1000, M - 3], [0, 1, M]):
        c.fill_(float("nan"))
        B.lcma_i8_gemm_experts(Aq, sa, torch.tensor(offsets, dtype=torch.int32, device="cuda"), Wq, one, c, 0, bias)
        a, b = offsets[1:]
        assert (c[:a] == 3).all().item() and (c[a:b] == 5).all().item() and (c[b:] == 0).all().item()


def test_very_many_long_rows_quantised():
    """2^22 rows of more than 4096 values: more threads than a launch holds along one dimension."""
    import torch
    from paper_2605_06057_amd import binding as B
    rows, K = (1 << 22) + 5, 4104
    x = torch.zeros((rows, K), dtype=torch.bfloat16, device="cuda")
    number = torch.arange(rows, device="cuda") % 100 + 27
    x[:, 1], x[:, K - 1] = number, -number
    Q, S = B.lcma_i8_quantize(x)
    del x
    assert torch.equal(S.cpu(), number.cpu().float() / torch.tensor(127.0))  # (a division; torch multiplies by 1 / 127 on the GPU)
    for k, code in ((1, 127), (K - 1, -127), (0, 0), (K, 0)):
        assert (Q[:, k] == code).all().item()


def test_one_row_whose_stride_says_nothing():
    """A single row of a tensor with rows of 2^30 elements, which no row that is there is apart from another."""
    import torch
    from paper_2605_06057_amd import binding as B
    rng = np.random.default_rng(1)
    stored, x = _values(rng, (1, 200), "bf16")
    dev = _device(stored, "bf16")
    Q, S = B.lcma_i8_quantize(dev.as_strided((1, 200), (1 << 30, 1)))
    q, s = X.i8_quantize(x)
    assert np.array_equal(Q.cpu().numpy()[:, :200], q) and np.array_equal(S.cpu().numpy(), s)
    Wq, w = _codes(rng, (), 33, 200)
    c = torch.empty((33,), device="cuda")
    B.lcma_i8_gemm_nt(Q, S, Wq, torch.ones((33,), device="cuda"), c.as_strided((1, 33), (1 << 30, 1)), 200)
    _check(c.cpu().numpy().astype(np.float64)[None], X.i8_gemm(q, s, w, np.ones(33, np.float32)), "f32", None)
