"""examples/experts_layer.py: the served layer against the definition of its steps in 64 bits, the trained one's gradients against those of plain autograd."""
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


@pytest.mark.parametrize("tokens,top,experts,hidden,ffn", [(1, 1, 2, 64, 40), (37, 2, 5, 136, 72), (300, 3, 7, 256, 200)])
def test_served(layer, tokens, top, experts, hidden, ffn):
    """Both products round their result to bf16 (2^-9 of a value, rms), which moves codes of the second quantisation by a step now and then; a step is 1/127 of a row's
    largest value.  Held to 2 % of the result, about three times what such moves add up to."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    normal = lambda *s: torch.randn(s, device="cuda", generator=gen).bfloat16()
    x, w_in, w_out = normal(tokens, hidden), normal(experts, 2 * ffn, hidden) * 0.1, normal(experts, hidden, ffn) * 0.1
    ids, w = layer.route(x, normal(experts, hidden), top)
    ids[0, 0] = -1
    got = layer.ServedExperts(w_in, w_out)(x, ids, w).double().cpu().numpy()
    host = lambda t: t.double().cpu().numpy()
    order, position, offsets = X.tokens_sort(ids.cpu().numpy(), experts)
    flat = lambda v: [X.i8_quantize(host(m)) for m in v]
    win, wout = flat(w_in), flat(w_out)
    stack = lambda p: (np.stack([q for q, _ in p]), np.stack([s for _, s in p]))
    q, s = X.i8_quantize(X.tokens_dispatch(host(x), position))
    h = X.i8_gemm_experts(q, s, offsets, *stack(win))
    q, s = X.i8_quantize(X.silu_gate(h))
    y = X.i8_gemm_experts(q, s, offsets, *stack(wout))
    want = X.tokens_combine(y, position, w.cpu().numpy())
    assert np.linalg.norm(got - want) <= 0.02 * np.linalg.norm(want)


def test_trained(layer):
    """fp32 throughout: products of the library and of torch in fp32 sums of at most 300 terms, so 1e-5 of each gradient's norm."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(3)
    normal = lambda *s: torch.randn(s, device="cuda", generator=gen)
    T, top, E, H, F = 300, 2, 5, 64, 48
    x, w, ids = normal(T, H), normal(E, F, H), torch.randint(-1, E, (T, top), device="cuda", generator=gen).int()
    weights, up = torch.rand((T, top), device="cuda", generator=gen), normal(T, F)
    mine = [t.clone().requires_grad_() for t in (x, w, weights)]
    layer.TrainedLinearExperts.apply(mine[0], mine[1], ids, mine[2]).backward(up)
    ref = [t.double().clone().requires_grad_() for t in (x, w, weights)]
    every = torch.einsum("th,efh->tef", ref[0], ref[1])
    picked = every[torch.arange(T, device="cuda")[:, None], ids.clamp(min=0).long()] * (ids >= 0)[:, :, None]
    (picked * ref[2][:, :, None]).sum(1).backward(up.double())
    for a, b in zip(mine, ref):
        assert ((a.grad.double() - b.grad).norm() / b.grad.norm()).item() <= 1e-5


def test_training_reduces_the_loss(layer):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(4)
    normal = lambda *s: torch.randn(s, device="cuda", generator=gen)
    x, target, w = normal(512, 128).bfloat16(), (normal(512, 64) * 0.1).bfloat16(), (normal(4, 64, 128) * 0.09).bfloat16()
    losses = layer.train(x, target, w, normal(4, 128) * 0.1, 2, 6)
    assert all(b < a for a, b in zip(losses, losses[1:])), losses


def test_training_leaves_its_arguments_alone(layer):
    """In fp32, where the weights could be their own fp32 copies."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(5)
    normal = lambda *s: torch.randn(s, device="cuda", generator=gen)
    args = [normal(256, 64), normal(256, 64) * 0.1, normal(4, 64, 64) * 0.09, normal(4, 64) * 0.1]
    before = [t.clone() for t in args]
    losses = layer.train(*args, 2, 4)
    assert all(torch.equal(a, b) and not a.requires_grad for a, b in zip(args, before)) and all(b < a for a, b in zip(losses, losses[1:])), losses
