"""lcma_gemm_experts_grad of matrices whose columns do not fill their rows: widths that are no whole dwords or no whole 16 bytes in rows of whole 16 bytes (which the kernels that load straight into LDS
take), and in rows of whole dwords.  Whole numbers of -4 .. 4: every fp32 sum is exact and dW is the exact result rounded once."""
import numpy as np
import pytest

from oracle import experts as X

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch, {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _lib():
    from paper_2605_06057_amd import binding
    return binding


@pytest.fixture(params=["", "any64x64", "any128x128", "64x64", "64x128", "256x256"], scope="module")
def kernel(request):
    _lib().lcma_set_tuning("experts_kernel", request.param)
    yield request.param
    _lib().lcma_set_tuning("experts_kernel", "")


def _rows(gen, rows, width, pitch, dtype):
    """rows x width whole numbers in rows of `pitch` elements with NaN behind, the last row without them."""
    torch, types = _torch()
    flat = torch.full((rows * pitch,), float("nan"), device="cuda", dtype=types[dtype])
    out = flat[: (rows - 1) * pitch + width].as_strided((rows, width), (pitch, 1))
    out.copy_(torch.randint(-4, 5, (rows, width), device="cuda", generator=gen))
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("counts", [[700], [1], [64, 0, 65, 3], [128, 63]], ids=str)
@pytest.mark.parametrize("N,ldn,K,ldk", [(257, 264, 129, 136), (257, 264, 130, 132), (1, 8, 7, 8), (63, 64, 65, 72), (130, 136, 258, 264), (255, 256, 320, 320), (64, 72, 127, 128), (66, 66, 34, 34), (511, 512, 513, 520)])
def test_columns_that_do_not_fill_their_rows(kernel, N, ldn, K, ldk, counts, dtype):
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(N + K + len(counts))
    rows, E = sum(counts), len(counts)
    dc, a = _rows(gen, rows, N, ldn, dtype), _rows(gen, rows, K, ldk, dtype)
    offsets = torch.tensor(np.cumsum([0] + counts), dtype=torch.int32, device="cuda")
    room = torch.full((E + 2, N, K), 99.0, device="cuda").to(types[dtype])
    _lib().lcma_gemm_experts_grad(dc, a, offsets, room[1:-1])
    want = X.gemm_experts_grad(dc.double().cpu().numpy(), a.double().cpu().numpy(), offsets.cpu().numpy())
    assert np.array_equal(room[1:-1].double().cpu().numpy(), torch.from_numpy(want).float().to(types[dtype]).double().numpy())
    assert (room[0] == 99.0).all() and (room[-1] == 99.0).all()
