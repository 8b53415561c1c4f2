"""Products with more tiles than one launch has work-groups for (2^22): several launches, every tile once, rows behind the last expert's zero."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def freed():
    yield
    import torch
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,rows", [("bfloat16", (1 << 28) + 100), ("float32", (1 << 26) + 100)])
def test_4_bit_weights_in_several_launches(dtype, rows):
    """One column, K = 1: C = X q S with q S of a few bits, exact."""
    import torch
    from paper_2605_06057_amd import binding as L
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randint(-8, 9, (rows, 1), device="cuda", generator=gen, dtype=torch.int8).to(getattr(torch, dtype))
    room = torch.full((rows + 2, 1), 9.0, device="cuda", dtype=x.dtype)
    one = lambda v: L.lcma_i4_prepare(torch.tensor([[v]], dtype=torch.int8, device="cuda"), torch.full((1, 1), 0.5, device="cuda"), 64)
    L.lcma_i4_gemm_nt(x, one(5), room[1:-1], 64)
    assert torch.equal(room[1:-1], x * 2.5) and (room[0] == 9.0).all() and (room[-1] == 9.0).all()
    room.fill_(9.0)
    ends = [0, 7, 7, rows // 2 + 1, rows - 50]
    L.lcma_i4_gemm_experts(x, torch.tensor(ends, dtype=torch.int32, device="cuda"), torch.stack([one(v) for v in (2, 3, -4, 7)]), room[1:-1], 64)
    for e, q in enumerate((2, 3, -4, 7)):
        assert torch.equal(room[1 + ends[e]:1 + ends[e + 1]], x[ends[e]:ends[e + 1]] * (q * 0.5))
    assert (room[1 + ends[-1]:-1] == 0).all() and (room[0] == 9.0).all() and (room[-1] == 9.0).all()


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("b_nk", [True, False])
def test_experts_products_in_several_launches(dtype, b_nk):
    import torch
    from paper_2605_06057_amd import binding as L
    gen = torch.Generator(device="cuda").manual_seed(2)
    rows, q = (1 << 29) + 1000, (2.0, 3.0, -4.0, 7.0)
    x = torch.randint(-8, 9, (rows, 1), device="cuda", generator=gen, dtype=torch.int8).to(getattr(torch, dtype))
    room = torch.full((rows + 2, 1), 9.0, device="cuda", dtype=x.dtype)
    ends = [0, 7, 7, rows // 2 + 1, rows - 50]
    L.lcma_gemm_experts(x, torch.tensor(ends, dtype=torch.int32, device="cuda"), torch.tensor(q, device="cuda", dtype=x.dtype).view(4, 1, 1), room[1:-1], b_nk)
    for e in range(4):
        assert torch.equal(room[1 + ends[e]:1 + ends[e + 1]], x[ends[e]:ends[e + 1]] * q[e])
    assert (room[1 + ends[-1]:-1] == 0).all() and (room[0] == 9.0).all() and (room[-1] == 9.0).all()


@pytest.mark.parametrize("wide", ["K", "N"])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_weights_gradients_in_several_launches(dtype, wide):
    """Three experts, the middle one without rows; whole numbers."""
    import torch
    from paper_2605_06057_amd import binding as L
    gen = torch.Generator(device="cuda").manual_seed(3)
    n = (1 << 29) - 1
    few = lambda *s: torch.randint(-4, 5, s, device="cuda", generator=gen, dtype=torch.int8).to(getattr(torch, dtype))
    long, short = few(3, n), few(3, 1)
    room = torch.full((3 * n + 2,), 9.0, device="cuda", dtype=long.dtype)
    dw = room[1:-1].view((3, 1, n) if wide == "K" else (3, n, 1))
    offsets = torch.tensor([0, 2, 2, 3], dtype=torch.int32, device="cuda")
    L.lcma_gemm_experts_grad(*((short, long) if wide == "K" else (long, short)), offsets, dw)
    assert torch.equal(dw[0].view(-1), long[0] * short[0] + long[1] * short[1])
    assert not dw[1].any() and torch.equal(dw[2].view(-1), long[2] * short[2]) and room[0] == 9.0 and room[-1] == 9.0
