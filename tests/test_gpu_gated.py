"""lcma_gated_silu and its gradient against the definitions in 64 bits.

Arithmetic in fp32: the exponential is good to 2^-22 of its value (its argument is held in two parts; the instruction itself to 2^-23), the reciprocal to 2^-23, each of
up to six products and sums to 2^-24: 2^-21 of the product of the factors' magnitudes in all.  The slope s (1 + g (1 - s)) is a sum of two terms: off by 2^-21 of
s (1 + |g| (1 - s)).  Then half a step of the result's type, or of its smallest number."""
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


def _tolerance(t, want, magnitude):
    torch, types = _torch()
    f = torch.finfo(types[t])
    return f.eps / 2 * np.abs(want) + 2.0 ** -21 * magnitude * (1 + f.eps) + f.smallest_normal * f.eps


def _check(dy, x, y, dx, t):
    host = lambda v: v.double().cpu().numpy()
    dyn, xn = host(dy), host(x)
    with np.errstate(over="ignore"):
        want, back = X.silu_gate(xn), X.silu_gate_grad(dyn, xn)
        g, u = np.split(xn, 2, axis=1)
        s = 1 / (1 + np.exp(-g))
    most = np.concatenate([np.abs(dyn * u) * s * (1 + np.abs(g) * (1 - s)), np.abs(dyn * g) * s], axis=1)
    assert (np.abs(host(y) - want) <= _tolerance(t, want, np.abs(want))).all()
    assert (np.abs(host(dx) - back) <= _tolerance(t, back, most)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,F,pad", [(1, 1, 0), (3, 8, 0), (2, 2048, 0), (5, 77, 3), (1, 14336, 0), (300, 264, 8), (1029, 1000, 0), (7, 2056, 5), (64, 16, 0)])
def test_values_and_gradient(rows, F, pad, dtype):
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(rows + F)
    normal = lambda n, w: torch.randn((n, w), device="cuda", generator=gen).to(types[dtype])
    x, dy = (2 * normal(rows, 2 * F + pad))[:, : 2 * F], normal(rows, F + pad)[:, :F]
    new = lambda w: torch.full((rows + 1, w + pad), 7.0, device="cuda").to(types[dtype])
    yw, dxw = new(F), new(2 * F)
    L = _lib()
    y, dx = L.lcma_gated_silu(x, yw[:rows, :F]), L.lcma_gated_silu_grad(dy, x, dxw[:rows, : 2 * F])
    _check(dy, x, y, dx, dtype)
    assert (yw[:, F:] == 7.0).all() and (dxw[:, 2 * F:] == 7.0).all() and (yw[rows:] == 7.0).all() and (dxw[rows:] == 7.0).all()
    assert torch.equal(L.lcma_gated_silu(x), y) and torch.equal(L.lcma_gated_silu_grad(dy, x), dx)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gates_far_from_zero(dtype):
    """Gates from -170 to 200 with linear parts and gradients that bring small values back into range."""
    torch, types = _torch()
    g = torch.linspace(-170, 200, 1480, device="cuda").to(types[dtype])
    for up in (1.0, 1e30):
        x = torch.cat([g, torch.full_like(g, up)])[None]
        for down in (1.0, 1e-4):
            dy = torch.full_like(g, down)[None]
            L = _lib()
            y, dx = L.lcma_gated_silu(x), L.lcma_gated_silu_grad(dy, x)
            _check(dy, x, y, dx, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_gradient_against_differences(dtype):
    """Central differences of the 64-bit definition, h = 2^-12: off by h^2 / 6 of the third derivative, which is below 1 for silu, times |u dy|, beside the rounding of the result."""
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(5)
    x, dy = torch.randn((4, 64), device="cuda", generator=gen).to(types[dtype]), torch.randn((4, 32), device="cuda", generator=gen).to(types[dtype])
    got = _lib().lcma_gated_silu_grad(dy, x).double().cpu().numpy()
    xn, dyn, h = x.double().cpu().numpy(), dy.double().cpu().numpy(), 2.0 ** -12
    for i in range(64):
        step = np.zeros_like(xn)
        step[:, i] = h
        want = ((X.silu_gate(xn + step) - X.silu_gate(xn - step)) * dyn).sum(axis=1) / (2 * h)
        slack = h * h * np.abs(dyn).max() * np.abs(xn).max() + 2.0 ** -20 * np.abs(xn).max() * np.abs(dyn).max()
        assert (np.abs(got[:, i] - want) <= torch.finfo(types[dtype]).eps / 2 * np.abs(want) + slack).all()


def test_special_gates():
    """A NaN stays in its element; a gate of +infinity gives an infinite value; zeros give zeros."""
    torch, types = _torch()
    inf, nan = float("inf"), float("nan")
    x = torch.tensor([[nan, inf, 0.0, -200.0, 1.0, 1.0, 2.0, 3.0, 1.0, nan]], device="cuda")
    L = _lib()
    y, dx = L.lcma_gated_silu(x)[0], L.lcma_gated_silu_grad(torch.ones((1, 5), device="cuda"), x)[0]
    assert y[0].isnan() and y[1] == inf and y[2] == 0 and y[3] == 0 and y[4].isnan()
    assert dx[0].isnan() and dx[2] == 0.5 * 3.0 and dx[3] == 0 and dx[4].isnan() and dx[7] == 0 and dx[8] == 0 and abs(dx[9].item() - 0.7310586) < 1e-6


def test_captured_and_replayed():
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, dy = torch.randn((50, 400), device="cuda", generator=gen).bfloat16(), torch.randn((50, 200), device="cuda", generator=gen).bfloat16()
    L = _lib()
    run = lambda: (L.lcma_gated_silu(x), L.lcma_gated_silu_grad(dy, x))
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for _ in range(3):
        x.normal_(generator=gen)
        want = run()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_empty():
    torch, types = _torch()
    L = _lib()
    assert L.lcma_gated_silu(torch.empty((0, 8), device="cuda")).shape == (0, 4) and L.lcma_gated_silu(torch.empty((3, 0), device="cuda")).shape == (3, 0)
    assert L.lcma_gated_silu_grad(torch.empty((0, 4), device="cuda"), torch.empty((0, 8), device="cuda")).shape == (0, 8)
