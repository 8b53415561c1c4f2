"""The experts' products, their gate and 4-bit weights where addresses pass 32 bits: rows, results and weights of more than 4 GiB; leading dimensions of megabytes; a stream of its own."""
import pytest

pytestmark = pytest.mark.gpu


def _lib():
    import torch
    from paper_2605_06057_amd import binding
    return torch, binding


@pytest.fixture(autouse=True)
def freed():
    yield
    _lib()[0].cuda.empty_cache()


def _signs(torch, gen, *shape):
    return (torch.randint(0, 2, shape, device="cuda", generator=gen, dtype=torch.int8) * 2 - 1).bfloat16()


@pytest.mark.parametrize("pad", [0, 3], ids=["whole 16 bytes", "off 16 bytes"])
def test_rows_and_results_beyond_4_gib(pad):
    """Values of -1 and 1, K sums of them: exact in fp32, and up to 256 in bf16 too; the gradient's are sums of up to 2^20 of them, rounded once."""
    torch, L = _lib()
    gen = torch.Generator(device="cuda").manual_seed(1)
    K, N, ends = 1024 + pad, 1032 + pad, [0, 1000000, 1000000, 2048000, 2200000]
    rows, E = ends[-1] + 5, len(ends) - 1
    a, w = _signs(torch, gen, rows, K), _signs(torch, gen, E, N, K)
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    c = L.lcma_gemm_experts(a, offsets, w)
    assert c.numel() * 2 > 1 << 32
    for e in range(E):
        for r in (ends[e], (ends[e] + ends[e + 1]) // 2, ends[e + 1] - 300):
            if ends[e] <= r and r + 300 <= ends[e + 1]:
                assert torch.equal(c[r:r + 300], (a[r:r + 300].float() @ w[e].float().t()).bfloat16())
    assert (c[ends[-1]:] == 0).all()
    d = _signs(torch, gen, rows, N)
    back = L.lcma_gemm_experts(d, offsets, w, b_nk=False)
    assert torch.equal(back[ends[3]:ends[3] + 300], (d[ends[3]:ends[3] + 300].float() @ w[3].float()).bfloat16())
    assert torch.equal(back[ends[4] - 300:ends[4]], (d[ends[4] - 300:ends[4]].float() @ w[3].float()).bfloat16())
    dw = L.lcma_gemm_experts_grad(d, a, offsets)
    for e in range(E):  # (whole numbers below 2^24: the blocks' sums are exact in fp32)
        want = torch.zeros((N, K), device="cuda")
        for r in range(ends[e], ends[e + 1], 1 << 17):
            s = slice(r, min(r + (1 << 17), ends[e + 1]))
            want += d[s].float().t().contiguous() @ a[s].float()
        assert torch.equal(dw[e], want.bfloat16())


@pytest.mark.parametrize("kernel", ["", "any64x64", "32x32", "64x128", "128x256", "256x256"])
def test_weights_beyond_4_gib(kernel):
    torch, L = _lib()
    gen = torch.Generator(device="cuda").manual_seed(2)
    E, N, K = 40, 8192, 8200
    w = torch.zeros((E, N, K), device="cuda", dtype=torch.bfloat16)
    w[-2:] = _signs(torch, gen, 2, N, K)
    offsets = torch.tensor([0] * (E - 1) + [30, 70], dtype=torch.int32, device="cuda")
    a, d = _signs(torch, gen, 70, K), _signs(torch, gen, 70, N)
    L.lcma_set_tuning("experts_kernel", kernel)
    try:
        c, back, dw = L.lcma_gemm_experts(a, offsets, w), L.lcma_gemm_experts(d, offsets, w, b_nk=False), L.lcma_gemm_experts_grad(d, a, offsets)
    finally:
        L.lcma_set_tuning("experts_kernel", "")
    for e, s in ((E - 2, slice(0, 30)), (E - 1, slice(30, 70))):
        assert torch.equal(c[s], (a[s].float() @ w[e].float().t()).bfloat16())
        assert torch.equal(back[s], (d[s].float() @ w[e].float()).bfloat16())
        assert torch.equal(dw[e], (d[s].float().t().contiguous() @ a[s].float()).bfloat16())
    assert all((dw[e] == 0).all() for e in range(E - 2))


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_leading_dimensions_of_megabytes(dtype):
    """Rows 2^23 bytes and more apart, which the kernels with 32-bit offsets do not take."""
    torch, L = _lib()
    gen = torch.Generator(device="cuda").manual_seed(3)
    rows, N, K, ld = 700, 72, 136, 1 << 22
    far = torch.empty((rows, ld), device="cuda", dtype=getattr(torch, dtype))
    a, c, d = far[:, :K], far[:, 1000:1000 + N], far[:, 5000:5000 + N]
    a.copy_(_signs(torch, gen, rows, K))
    d.copy_(_signs(torch, gen, rows, N))
    w, offsets = _signs(torch, gen, 3, N, K).to(a.dtype), torch.tensor([0, 300, 300, 690], dtype=torch.int32, device="cuda")
    own = torch.empty((rows, N), device="cuda", dtype=a.dtype)
    L.lcma_gemm_experts(a, offsets, w, own)
    back, dw = L.lcma_gemm_experts(d, offsets, w, b_nk=False), L.lcma_gemm_experts_grad(d, a, offsets)
    near = L.lcma_gemm_experts(a.contiguous(), offsets, w)
    assert torch.equal(own, near) and (own[690:] == 0).all()  # (whole numbers: every kernel gives the same)
    assert torch.equal(back, L.lcma_gemm_experts(d.contiguous(), offsets, w, b_nk=False)) and torch.equal(dw, L.lcma_gemm_experts_grad(d.contiguous(), a.contiguous(), offsets))
    assert torch.equal(own[:300].float(), a[:300].float() @ w[0].float().t())
    L.lcma_gemm_experts(a.contiguous(), offsets, w, c)
    assert torch.equal(c, near)


def test_4_bit_weights_and_rows_beyond_4_gib():
    torch, L = _lib()
    gen = torch.Generator(device="cuda").manual_seed(4)
    E, N, K = 70, 8192, 16384
    one = torch.randn((2, N, K), device="cuda", generator=gen).bfloat16()
    w = one[:1].repeat(E, 1, 1)
    w[-1] = one[1]
    wp = L.lcma_i4_quantize(w, 128)
    assert wp.numel() > 1 << 32
    pair = L.lcma_i4_quantize(one, 128)
    assert torch.equal(wp[0], pair[0]) and torch.equal(wp[-1], pair[1]) and torch.equal(wp[-2], pair[0])
    x = torch.randn((40, K), device="cuda", generator=gen).bfloat16()
    c, few = torch.empty((40, N), device="cuda", dtype=x.dtype), torch.empty((40, N), device="cuda", dtype=x.dtype)
    for kernel in ("16x16", "16x32", "16x64", "64x64"):
        L.lcma_set_tuning("i4_kernel", kernel)
        try:
            L.lcma_i4_gemm_experts(x, torch.tensor([0] * (E - 1) + [17, 40], dtype=torch.int32, device="cuda"), wp, c)
            L.lcma_i4_gemm_experts(x, torch.tensor([0, 17, 40], dtype=torch.int32, device="cuda"), pair, few)
        finally:
            L.lcma_set_tuning("i4_kernel", "")
        assert torch.equal(c, few)
    del w, wp
    rows = 70000  # 4.6 GB of results
    small, q = torch.randn((70, 64), device="cuda", generator=gen).bfloat16(), L.lcma_i4_quantize(torch.randn((32776, 64), device="cuda", generator=gen).bfloat16(), 32)
    x, c, want = small.repeat(rows // 70, 1), torch.empty((rows, 32776), device="cuda", dtype=small.dtype), torch.empty((70, 32776), device="cuda", dtype=small.dtype)
    for kernel in ("16x64", "64x64"):
        L.lcma_set_tuning("i4_kernel", kernel)
        try:
            L.lcma_i4_gemm_nt(x, q, c, 32)
            L.lcma_i4_gemm_nt(small, q, want, 32)
        finally:
            L.lcma_set_tuning("i4_kernel", "")
        assert all(torch.equal(c[r:r + 70], want) for r in (0, 35000, rows - 70))


def test_gate_beyond_4_gib():
    torch, L = _lib()
    gen = torch.Generator(device="cuda").manual_seed(5)
    rows, F = 200000, 8200
    part = torch.randn((1000, 2 * F), device="cuda", generator=gen).bfloat16()
    x, up = part.repeat(rows // 1000, 1), part[:, :F].repeat(rows // 1000, 1)
    y, dx = L.lcma_gated_silu(x), L.lcma_gated_silu_grad(up, x)
    want, grad = L.lcma_gated_silu(part), L.lcma_gated_silu_grad(part[:, :F], part)
    for r in (0, 131000, rows - 1000):
        assert torch.equal(y[r:r + 1000], want) and torch.equal(dx[r:r + 1000], grad)


def test_a_stream_of_its_own():
    """Calls behind slow work on another stream than the default one, whose results they need."""
    torch, L = _lib()
    gen = torch.Generator(device="cuda").manual_seed(6)
    E, N, K, rows = 4, 520, 264, 300
    w, base = _signs(torch, gen, E, N, K), _signs(torch, gen, rows, K)
    offsets = torch.tensor([0, 100, 120, 120, 290], dtype=torch.int32, device="cuda")
    want = L.lcma_gated_silu(L.lcma_gemm_experts(base, offsets, w))
    slow = torch.randn((8192, 8192), device="cuda", generator=gen)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a = torch.zeros_like(base)
        for _ in range(4):
            slow @ slow
        a.copy_(base)
        got = L.lcma_gated_silu(L.lcma_gemm_experts(a, offsets, w))
    side.synchronize()
    assert torch.equal(got, want)
