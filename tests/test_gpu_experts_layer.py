"""The experts' layer as a whole, as examples/experts_layer.py runs it: trained (its gradients against plain autograd in 64 bits, captured and replayed) and served with
4-bit weights (against the definition of its steps in 64 bits)."""
import importlib.util
import os

import numpy as np
import pytest

from oracle import experts as X

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def layer():
    spec = importlib.util.spec_from_file_location("experts_layer", os.path.join(ROOT, "examples", "experts_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _inputs(T, top, E, H, F, dtype, seed=3):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(s, device="cuda", generator=gen)
    x, w_in, w_out = normal(T, H).to(dtype), (normal(E, 2 * F, H) / H ** 0.5).to(dtype), (normal(E, H, F) / F ** 0.5).to(dtype)
    return x, w_in, w_out, torch.randint(-1, E, (T, top), device="cuda", generator=gen).int(), torch.rand((T, top), device="cuda", generator=gen), normal(T, H).to(dtype)


def _reference(x, w_in, w_out, ids, weights, up):
    """Plain autograd in 64 bits: the result, the four gradients, and for each token and choice the norm of what the expert gave."""
    import torch
    norms = torch.zeros(ids.shape, dtype=torch.float64, device=x.device)
    ref = [t.double().clone().requires_grad_() for t in (x, w_in, w_out, weights)]
    out = torch.zeros_like(ref[0])
    for e in range(w_in.shape[0]):
        t, j = (ids == e).nonzero(as_tuple=True)
        g, u = (ref[0][t] @ ref[1][e].t()).chunk(2, dim=1)
        y = (torch.nn.functional.silu(g) * u) @ ref[2][e].t()
        norms[t, j] = y.detach().norm(dim=1)
        out = out.index_add(0, t, ref[3][t, j, None] * y)
    out.backward(up.double())
    return [out.detach()] + [r.grad for r in ref], norms


# A rounding is off by 2^-8 (bf16), 2^-11 (fp16) of a value at most; over a binade its rms is 0.41 of that.  On the way to any gradient lie at most six (the gate and up rows, the gate, the
# product out, its gradient, the gate's, the result), independent, so sqrt(6) * 0.41 = 1.0 of that bound in the norm, and those before the gate grow by its slopes, less than twice: 2.
# fp32: the rounding is 2^-24, the sums have at most 700 products in any order, rms sqrt(700) * 2^-24 = 1.6e-6 of their terms' norm, four sums one behind the other: 1e-5.
# The router's weights' gradient is one product of vectors, up . y, for each token and expert: its error up . dy is at most |up| |dy| (Cauchy and Schwarz), whatever cancels in up . y,
# so it is held against |up| |y| instead of itself.
@pytest.mark.parametrize("dtype,tolerance", [("float32", 1e-5), ("bfloat16", 2 * 2.0 ** -8), ("float16", 2 * 2.0 ** -11)])
@pytest.mark.parametrize("T,top,E,H,F", [(300, 2, 5, 64, 48), (37, 3, 4, 72, 40), (5, 1, 3, 33, 21), (700, 2, 4, 264, 200)])
def test_trained(layer, T, top, E, H, F, dtype, tolerance):
    import torch
    x, w_in, w_out, ids, weights, up = _inputs(T, top, E, H, F, getattr(torch, dtype))
    mine = [t.clone().requires_grad_() for t in (x, w_in, w_out, weights)]
    out = layer.TrainedExperts.apply(mine[0], mine[1], mine[2], ids, mine[3])
    out.backward(up)
    want, y = _reference(x, w_in, w_out, ids, weights, up)
    norms = [b.norm() for b in want[:-1]] + [(up.double().norm(dim=1)[:, None] * y).norm()]
    for a, b, norm in zip([out] + [m.grad for m in mine], want, norms):
        assert ((a.double() - b).norm() / norm).item() <= tolerance


def test_a_captured_step_gives_the_eager_steps_bits(layer):
    """The calls of a step in a graph, replayed with new tokens and new routes in the same places."""
    import torch
    x, w_in, w_out, ids, weights, up = _inputs(200, 2, 6, 136, 72, torch.bfloat16)

    class Ctx:
        def save_for_backward(self, *t):
            self.saved_tensors = t

    def step():
        ctx = Ctx()
        out = layer.TrainedExperts.forward(ctx, x, w_in, w_out, ids, weights)
        return [out] + [g for g in layer.TrainedExperts.backward(ctx, up) if g is not None]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for seed in range(3):
        new = _inputs(200, 2, 6, 136, 72, torch.bfloat16, seed)
        for a, b in zip((x, w_in, w_out, ids, weights, up), new):
            a.copy_(b)
        eager = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, eager))


@pytest.mark.parametrize("tokens,top,experts,hidden,ffn,group", [(1, 1, 2, 64, 40, 32), (37, 2, 5, 136, 72, 64), (300, 3, 7, 256, 200, 128)])
def test_served_in_4_bits(layer, tokens, top, experts, hidden, ffn, group):
    """Against the steps' definitions in 64 bits on the same codes: four roundings to bf16 (the gate and up rows, the gate, the product out, the tokens), each 2^-8 of a value at most and
    0.41 of that in rms; sqrt(4) * 0.41 = 0.8, and the first grows by the gate's slopes, less than twice: 1.5 * 2^-8 of the result's norm."""
    import torch
    x, w_in, w_out, ids, weights, _ = _inputs(tokens, top, experts, hidden, ffn, torch.bfloat16, 7)
    ids[0, 0] = -1 if tokens > 1 else 0
    got = layer.ServedExperts4(w_in, w_out, group)(x, ids, weights).double().cpu().numpy()
    host = lambda t: t.double().cpu().numpy()
    order, position, offsets = X.tokens_sort(ids.cpu().numpy(), experts)
    four = lambda w: np.stack([X.i4_dequantize(*X.i4_quantize(m, group), group) for m in host(w)])
    h = X.gemm_experts(X.tokens_dispatch(host(x), position), offsets, four(w_in))
    y = X.gemm_experts(X.silu_gate(h), offsets, four(w_out))
    want = X.tokens_combine(y, position, weights.cpu().numpy())
    assert np.linalg.norm(got - want) <= 1.5 * 2.0 ** -8 * np.linalg.norm(want)
