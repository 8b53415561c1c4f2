"""The gradients of the experts' products against differences, where every result is a whole number below 256, which bf16 holds: no slack in any type."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kernel", ["", "any64x64", "16x16", "64x64", "256x256"])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
def test_gradients_are_the_differences(dtype, kernel):
    """sum(C * up) is linear in A and in W: 1 more in one element changes it by the gradient.  Inputs of -1, 0 and 1: C up to 40, its gradients up to 24 and 20."""
    import torch
    from paper_2605_06057_amd import binding as L
    gen = torch.Generator(device="cuda").manual_seed(3)
    few = lambda *s: torch.randint(-1, 2, s, device="cuda", generator=gen).to(getattr(torch, dtype))
    a, w, up = few(34, 40), few(4, 24, 40), few(34, 24)
    offsets = torch.tensor([0, 5, 5, 14, 34], dtype=torch.int32, device="cuda")
    L.lcma_set_tuning("experts_kernel", kernel)
    try:
        value = lambda a_, w_: (L.lcma_gemm_experts(a_, offsets, w_).double() * up.double()).sum().item()
        da, dw, base = L.lcma_gemm_experts(up, offsets, w, b_nk=False), L.lcma_gemm_experts_grad(up, a, offsets), value(a, w)
        for r, k in [(0, 0), (4, 39), (5, 7), (13, 1), (14, 2), (33, 20)]:
            b = a.clone()
            b[r, k] += 1
            assert value(b, w) - base == da[r, k].item()
        for e, n, k in [(0, 0, 0), (0, 23, 39), (1, 3, 3), (2, 23, 39), (3, 10, 1)]:
            b = w.clone()
            b[e, n, k] += 1
            assert value(a, b) - base == dw[e, n, k].item()
        assert np.abs(da.double().cpu().numpy()).max() > 1 and dw.double().abs().max() > 1
    finally:
        L.lcma_set_tuning("experts_kernel", "")
