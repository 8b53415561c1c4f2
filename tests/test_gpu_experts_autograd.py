"""What autograd may ask of the experts' layers of examples/experts_layer.py beside the gradients themselves: some of them alone, and second derivatives, which there are none of."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def layer():
    spec = importlib.util.spec_from_file_location("experts_layer_autograd", os.path.join(ROOT, "examples", "experts_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _call(layer, name, needs):
    """The layer's result on leaves of which `needs` says which have a gradient (x, matrices, weights), and these."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(2)
    normal = lambda *s: torch.randn(s, device="cuda", generator=gen)
    matrices = [normal(4, 48, 40), normal(4, 40, 24)] if name == "TrainedExperts" else [normal(4, 32, 40)]
    ids = torch.randint(-1, 4, (30, 2), device="cuda", generator=gen).int()
    leaves = [normal(30, 40)] + matrices + [torch.rand((30, 2), device="cuda", generator=gen)]
    for t, n in zip(leaves, needs):
        t.requires_grad_(n)
    return getattr(layer, name).apply(*leaves[:-1], ids, leaves[-1]), leaves


CASES = [("TrainedLinearExperts", n) for n in ((1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 0, 1))] + [
    ("TrainedExperts", n) for n in ((1, 1, 1, 1), (1, 0, 0, 0), (0, 1, 0, 0), (0, 0, 1, 0), (0, 0, 0, 1), (1, 0, 0, 1))]


@pytest.mark.parametrize("name,needs", CASES, ids=str)
def test_gradients_that_are_not_asked_for_are_not_computed(layer, name, needs, monkeypatch):
    import torch
    everything, all_leaves = _call(layer, name, [True] * len(needs))
    torch.autograd.backward(everything, torch.ones_like(everything))
    grads, real = [], layer.lcma.lcma_gemm_experts_grad
    monkeypatch.setattr(layer.lcma, "lcma_gemm_experts_grad", lambda *a: grads.append(1) or real(*a))
    out, leaves = _call(layer, name, [bool(n) for n in needs])
    torch.autograd.backward(out, torch.ones_like(out))
    for t, full, n in zip(leaves, all_leaves, needs):
        assert torch.equal(t.grad, full.grad) if n else t.grad is None
    assert len(grads) == sum(needs[1:-1])


@pytest.mark.parametrize("name", ["TrainedLinearExperts", "TrainedExperts"])
@pytest.mark.parametrize("square", [False, True])
def test_a_second_derivative_is_refused(layer, name, square):
    """It would be taken for zero wherever the layer has part in it."""
    import torch
    out, leaves = _call(layer, name, [True] * (3 if name == "TrainedLinearExperts" else 4))
    with pytest.raises(RuntimeError, match="second derivative"):
        grad, = torch.autograd.grad((out.square() if square else out).sum(), leaves[0], create_graph=True)
        (grad * leaves[0]).sum().backward()
