"""4-bit weights without rows or columns."""
import pytest

pytestmark = pytest.mark.gpu


def test_weights_without_rows_or_columns():
    """One matrix or several, from values and from codes, as every other call takes them."""
    import torch
    from paper_2605_06057_amd import binding as L
    for lead in ((), (1,), (3,)):
        for N, K in ((0, 8), (5, 0), (0, 0)):
            w = torch.empty((*lead, N, K), device="cuda")
            assert L.lcma_i4_quantize(w, 32).shape == (*lead, 0)
            assert L.lcma_i4_prepare(w.to(torch.int8), torch.empty((*lead, N, -(-K // 32)), device="cuda"), 32).shape == (*lead, 0)
