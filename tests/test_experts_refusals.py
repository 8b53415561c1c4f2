"""What the 8-bit-integer product and the tokens' calls refuse, found out on the CPU: every refusal comes before anything is launched, so any
aligned address stands for a matrix.  A refusal has its status and names the call."""
import os

import pytest

A = 1 << 32  # addresses far apart
AT = {k: A * (i + 1) for i, k in enumerate(["x", "q", "s", "w", "sw", "bias", "c", "offsets", "position", "ids", "order", "weights", "dw", "dy", "space"])}


@pytest.fixture(scope="module")
def B():
    from paper_2605_06057_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2605_06057_amd import build
        build.build()
    binding.lib()
    return binding


CALLS = {
    "lcma_i8_quantize": dict(rows=4, K=100, X=AT["x"], ldx=100, dtype=1, gated=0, Q=AT["q"], S=AT["s"], stream=None),
    "lcma_i8_quantize_dispatch": dict(tokens=4, K=100, X=AT["x"], ldx=100, dtype=1, top_k=2, position=AT["position"], Q=AT["q"], S=AT["s"], stream=None),
    "lcma_i8_gemm_nt": dict(M=4, N=50, K=100, Aq=AT["q"], Sa=AT["s"], Wq=AT["w"], Sw=AT["sw"], bias=AT["bias"], C=AT["c"], ldc=50, dtype=1, stream=None),
    "lcma_i8_gemm_experts": dict(rows=4, N=50, K=100, experts=3, offsets=AT["offsets"], Aq=AT["q"], Sa=AT["s"], Wq=AT["w"], Sw=AT["sw"], bias=AT["bias"], C=AT["c"], ldc=50,
                                 dtype=1, stream=None),
    "lcma_tokens_sort": dict(tokens=3000, top_k=2, experts=3, ids=AT["ids"], order=AT["order"], position=AT["position"], offsets=AT["offsets"], workspace=AT["space"],
                             workspace_bytes=64, stream=None),
    "lcma_tokens_dispatch": dict(tokens=4, top_k=2, H=100, X=AT["x"], ldx=100, dtype=1, position=AT["position"], Y=AT["c"], ldy=100, stream=None),
    "lcma_tokens_combine": dict(tokens=4, top_k=2, H=100, Y=AT["x"], ldy=100, dtype=1, position=AT["position"], weights=AT["weights"], X=AT["c"], ldx=100, stream=None),
    "lcma_tokens_combine_grad": dict(tokens=4, top_k=2, H=100, dX=AT["x"], lddx=100, Y=AT["c"], ldy=100, dtype=1, position=AT["position"], weights=AT["weights"], dY=AT["dy"],
                                     lddy=100, dweights=AT["dw"], stream=None),
}
BAD = {
    "lcma_i8_quantize": [("DTYPE", dict(dtype=3)), ("ARG", dict(rows=-1)), ("ARG", dict(K=-1)), ("ARG", dict(X=None)), ("ARG", dict(Q=None)), ("ARG", dict(S=None)), ("ARG", dict(ldx=99)),
                         ("ARG", dict(gated=1)), ("ARG", dict(X=AT["x"] + 1)), ("ARG", dict(Q=AT["q"] + 8)), ("ARG", dict(S=AT["s"] + 2)), ("ARG", dict(Q=AT["x"] + 688)),
                         ("ARG", dict(S=AT["q"] + 508)), ("ARG", dict(S=AT["x"])), ("SHAPE", dict(K=131072, ldx=131072)), ("SHAPE", dict(rows=1 << 31)), ("SHAPE", dict(ldx=1 << 29))],
    "lcma_i8_quantize_dispatch": [("ARG", dict(position=None)), ("ARG", dict(top_k=0)), ("ARG", dict(position=AT["position"] + 1)), ("ARG", dict(position=AT["q"] + 1000)),
                                  ("ARG", dict(position=AT["s"])), ("SHAPE", dict(tokens=1 << 30))],
    "lcma_i8_gemm_nt": [("DTYPE", dict(dtype=-1)), ("ARG", dict(M=-1)), ("ARG", dict(N=-4)), ("ARG", dict(K=-4)), ("ARG", dict(ldc=49)), ("SHAPE", dict(K=131072)), ("SHAPE", dict(ldc=1 << 29))] +
                       [("ARG", {k: None}) for k in ("Aq", "Sa", "Wq", "Sw", "C")] + [("ARG", dict(Aq=AT["q"] + 4)), ("ARG", dict(Wq=AT["w"] + 8)), ("ARG", dict(Sa=AT["s"] + 1)),
                        ("ARG", dict(bias=AT["bias"] + 2)), ("ARG", dict(C=AT["c"] + 1)), ("ARG", dict(C=AT["w"] + 6398)), ("ARG", dict(C=AT["q"])), ("ARG", dict(C=AT["bias"] + 198)),
                        ("SHAPE", dict(M=1 << 31)), ("SHAPE", dict(M=(1 << 31) - 1, N=1 << 20, ldc=1 << 20, C=1 << 60))],
    "lcma_i8_gemm_experts": [("ARG", dict(experts=0)), ("SHAPE", dict(experts=1025)), ("ARG", dict(offsets=None)), ("ARG", dict(offsets=AT["offsets"] + 2)), ("ARG", dict(C=AT["offsets"] + 14)),
                             ("ARG", dict(C=AT["w"] + 128 * 149))],
    "lcma_tokens_sort": [("ARG", dict(tokens=-1)), ("ARG", dict(top_k=0)), ("ARG", dict(experts=0)), ("SHAPE", dict(experts=1025)), ("SHAPE", dict(tokens=1 << 30)), ("ARG", dict(workspace_bytes=63)),
                         ("ARG", dict(workspace=None)), ("ARG", dict(order=AT["ids"] + 23996)), ("ARG", dict(offsets=AT["space"] + 60)), ("ARG", dict(position=AT["position"] + 1))] +
                        [("ARG", {k: None}) for k in ("ids", "order", "position", "offsets")],
    "lcma_tokens_dispatch": [("DTYPE", dict(dtype=9)), ("ARG", dict(tokens=-1)), ("ARG", dict(H=-1)), ("ARG", dict(top_k=0)), ("ARG", dict(X=None)), ("ARG", dict(Y=None)), ("ARG", dict(position=None)),
                             ("ARG", dict(ldx=99)), ("ARG", dict(ldy=99)), ("ARG", dict(Y=AT["x"] + 798)), ("ARG", dict(X=AT["x"] + 1)), ("SHAPE", dict(tokens=1 << 30)),
                             ("SHAPE", dict(H=1 << 28, ldx=1 << 28, ldy=1 << 28))],
    "lcma_tokens_combine": [("DTYPE", dict(dtype=9)), ("ARG", dict(X=None)), ("ARG", dict(Y=None)), ("ARG", dict(position=None)), ("ARG", dict(ldx=99)), ("ARG", dict(ldy=99)),
                            ("ARG", dict(X=AT["x"] + 1598)), ("ARG", dict(X=AT["weights"] + 30)), ("ARG", dict(weights=AT["weights"] + 1)), ("SHAPE", dict(tokens=1 << 30))],
    "lcma_tokens_combine_grad": [("DTYPE", dict(dtype=9)), ("ARG", dict(weights=None)), ("ARG", dict(dweights=None)), ("ARG", dict(dX=None)), ("ARG", dict(Y=None)), ("ARG", dict(dY=None)),
                                 ("ARG", dict(lddx=99)), ("ARG", dict(ldy=99)), ("ARG", dict(lddy=99)), ("ARG", dict(dY=AT["c"] + 1598)), ("ARG", dict(dY=AT["x"])), ("ARG", dict(dweights=AT["weights"] + 28)),
                                 ("ARG", dict(dweights=AT["dy"] + 4)), ("ARG", dict(dweights=AT["dw"] + 1)), ("SHAPE", dict(tokens=1 << 30))],
}


@pytest.mark.parametrize("name,status,change", [(n, s, c) for n, cases in BAD.items() for s, c in cases], ids=lambda v: str(v)[:40])
def test_refusals(B, name, status, change):
    args = {**CALLS[name], **change}
    got = getattr(B.lib(), name)(*args.values())
    assert B.STATUS_NAMES[got] == "ERR_" + status
    assert B.lib().lcma_last_error().decode().startswith(name + ":")


@pytest.mark.parametrize("name,change", [("lcma_i8_quantize", dict(rows=0, X=None, Q=None, S=None)), ("lcma_i8_quantize_dispatch", dict(tokens=0, position=None, X=None, Q=None, S=None)),
                                         ("lcma_i8_gemm_nt", dict(M=0, C=None)), ("lcma_i8_gemm_nt", dict(N=0, C=None, Wq=None)), ("lcma_i8_gemm_experts", dict(rows=0, offsets=None, C=None)),
                                         ("lcma_tokens_dispatch", dict(tokens=0, X=None, Y=None, position=None)), ("lcma_tokens_dispatch", dict(H=0, X=None, Y=None)),
                                         ("lcma_tokens_combine", dict(tokens=0, X=None, Y=None, position=None)), ("lcma_tokens_combine", dict(H=0, X=None, Y=None)),
                                         ("lcma_tokens_combine_grad", dict(tokens=0, weights=None))], ids=lambda v: str(v)[:40])
def test_nothing_to_do_is_no_error(B, name, change):
    assert getattr(B.lib(), name)(*{**CALLS[name], **change}.values()) == B.LCMA_OK


def test_sizes(B):
    assert [B.lcma_i8_code_pitch(k) for k in (-1, 0, 1, 128, 129)] == [-1, 0, 128, 128, 256]
    size = B.lcma_tokens_sort_workspace_bytes
    assert size(0, 1, 8) == 0 and size(64, 2, 8) == 0 and size(-1, 1, 8) == size(1, 0, 8) == size(1, 1, 0) == size(1, 1, 1025) == size(1 << 30, 2, 8) == -1
    assert 0 <= size(1 << 20, 8, 64) < 1 << 22


def test_the_binding_refuses_what_it_cannot_pass_on(B):
    import torch
    x = torch.zeros((4, 8))
    with pytest.raises((AssertionError, ValueError)):
        B.lcma_i8_quantize(x)  # not on the GPU
    with pytest.raises((AssertionError, ValueError)):
        B.lcma_tokens_sort(torch.zeros((4, 2), dtype=torch.int32), 8)


def test_the_binding_names_the_argument_it_refuses(B):
    import torch
    calls = B._native()
    x, ids = torch.zeros((4, 8)), torch.zeros((4, 2), dtype=torch.int32)
    for f, args, what in [(calls.i8_quantize, (x, x, x, False), "X: expected a tensor on the GPU"), (calls.i8_quantize, (7, x, x, False), "X: expected a tensor"),
                          (calls.i8_quantize, (torch.zeros(4), x, x, False), "X: expected two dimensions"), (calls.tokens_sort, (ids, 0, ids, ids, ids, None), "experts: expected"),
                          (calls.tokens_dispatch, (x, ids, x), "X: expected a tensor on the GPU"), (calls.tokens_combine, (x, ids, None, x), "Y: expected a tensor on the GPU"),
                          (calls.i8_gemm_nt, (x, x, x, x, x, 8, None), "C: expected a tensor on the GPU")]:
        with pytest.raises(AssertionError, match=what):
            f(*args)
    with pytest.raises(TypeError):
        calls.i8_quantize(x)
    with pytest.raises(TypeError):
        calls.tokens_sort(ids, "three", ids, ids, ids, None)


def test_an_error_of_an_argument_is_passed_on(B):
    import torch

    class Neither:
        def __bool__(self):
            raise KeyError("neither")
    x = torch.zeros((4, 8))
    with pytest.raises(KeyError, match="neither"):
        B._native().i8_quantize(x, x, x, Neither())
