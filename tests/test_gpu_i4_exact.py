"""What the products with 4-bit weights may not lose: fp32 activations are multiplied with all of their bits.

A value of 19 bits times 24 + q (five bits) has 24, so that every term, their sums with -1.5 x and the result of a row with a single value are fp32 numbers: C is exact, to the bit."""
import numpy as np
import pytest

from oracle import experts as X

pytestmark = pytest.mark.gpu


def _lib():
    import torch
    from paper_2605_06057_amd import binding
    return torch, binding


@pytest.fixture(params=["", "16x16", "16x32", "16x64", "64x64"], scope="module")
def kernel(request):
    _lib()[1].lcma_set_tuning("i4_kernel", request.param)
    yield request.param
    _lib()[1].lcma_set_tuning("i4_kernel", "")


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("experts", [0, 3])
def test_all_bits_of_fp32_activations_count(kernel, experts, group):
    torch, L = _lib()
    gen = torch.Generator(device="cuda").manual_seed(group + experts)
    N, K, E = 48, 300, max(1, experts)
    number = lambda lo, hi, *s: torch.randint(lo, hi, s, device="cuda", generator=gen)
    codes = number(-8, 8, E, N, K).to(torch.int8)
    scales = torch.exp2(number(-6, 6, E, N, -(-K // group)).float())
    value = (2 * number(0, 1 << 17, K) + 1 + (1 << 18)).double() * torch.exp2(number(-28, -8, K).double()) * (2 * number(0, 2, K) - 1)  # odd 19-bit whole numbers, scaled
    x = torch.diag(value).float()
    c = torch.empty((K, N), device="cuda")
    if experts:
        ends = [0, 100, 100, 300]
        L.lcma_i4_gemm_experts(x, torch.tensor(ends, dtype=torch.int32, device="cuda"), L.lcma_i4_prepare(codes, scales, group), c, group)
    else:
        ends = [0, K]
        L.lcma_i4_gemm_nt(x, L.lcma_i4_prepare(codes[0], scales[0], group), c, group)
    host = lambda t: t.double().cpu().numpy()
    w = [X.i4_dequantize(host(codes[e]), host(scales[e]), group) for e in range(E)]
    want = np.concatenate([host(value)[a:b, None] * w[e].T[a:b] for e, (a, b) in enumerate(zip(ends, ends[1:]))])
    assert np.array_equal(host(c), want)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("K", [128, 1024, 2200])
@pytest.mark.parametrize("which", ["either sign", "one sign"])
def test_the_bound_that_the_header_states(kernel, which, K, group):
    """fp32: sums of a group off by up to 3 group 2^-20 of sum |X| 8 S (three parts of X, 2 group additions each, 2^-23 of a partial sum of up to 2 sum |X|, times 16 S); the groups' sums
    added in fp32, in any order of up to 2 for each (waves apart), 2^-23 of sum |X| 8 S each; the result."""
    torch, L = _lib()
    gen = torch.Generator(device="cuda").manual_seed(K + group)
    M, N = 17, 80
    codes = torch.randint(-8, 8, (N, K), device="cuda", generator=gen).to(torch.int8)
    codes[:20] = -8
    codes[20:40] = 7
    scales = torch.rand((N, -(-K // group)), device="cuda", generator=gen) * 0.02 + 0.001
    x = torch.randn((M, K), device="cuda", generator=gen)
    x = x.abs() if which == "one sign" else x
    c = L.lcma_i4_gemm_nt(x, L.lcma_i4_prepare(codes, scales, group), torch.empty((M, N), device="cuda"), group)
    host = lambda t: t.double().cpu().numpy()
    want = host(x) @ X.i4_dequantize(host(codes), host(scales), group).T
    terms = np.abs(host(x)) @ np.repeat(host(scales), group, axis=1)[:, :K].T * 8
    assert (np.abs(host(c) - want) <= (3 * group * 2.0 ** -20 + 2 * scales.shape[1] * 2.0 ** -23) * terms + 2.0 ** -24 * np.abs(want)).all()
