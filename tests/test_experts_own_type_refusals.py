"""What the experts' products in their own type, their gate and the calls with 4-bit weights refuse, found out on the CPU: every refusal comes before anything is launched,
so any aligned address stands for a matrix.  A refusal has its status and names the call."""
import os

import pytest

A = 1 << 40  # addresses far apart
AT = {k: A * (i + 1) for i, k in enumerate(["a", "w", "c", "offsets", "q", "s", "bias", "dy", "codes"])}


@pytest.fixture(scope="module")
def B():
    from paper_2605_06057_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2605_06057_amd import build
        build.build()
    binding.lib()
    return binding


CALLS = {
    "lcma_gemm_experts": dict(b_layout=2, rows=4, N=50, K=100, experts=3, offsets=AT["offsets"], A=AT["a"], lda=100, B=AT["w"], C=AT["c"], ldc=50, dtype=1, stream=None),
    "lcma_gemm_experts_grad": dict(rows=4, N=50, K=100, experts=3, offsets=AT["offsets"], dC=AT["c"], lddc=50, A=AT["a"], lda=100, dW=AT["w"], dtype=1, stream=None),
    "lcma_gated_silu": dict(rows=4, F=50, X=AT["a"], ldx=100, Y=AT["c"], ldy=50, dtype=1, stream=None),
    "lcma_gated_silu_grad": dict(rows=4, F=50, dY=AT["dy"], lddy=50, X=AT["a"], ldx=100, dX=AT["c"], lddx=100, dtype=1, stream=None),
    "lcma_i4_quantize": dict(experts=2, N=50, K=100, group=64, W=AT["w"], ldw=100, dtype=1, Wp=AT["q"], stream=None),
    "lcma_i4_prepare": dict(experts=2, N=50, K=100, group=64, codes=AT["codes"], scales=AT["s"], Wp=AT["q"], stream=None),
    "lcma_i4_gemm_nt": dict(M=4, N=50, K=100, group=64, X=AT["a"], ldx=100, Wp=AT["q"], bias=AT["bias"], C=AT["c"], ldc=50, dtype=1, stream=None),
    "lcma_i4_gemm_experts": dict(rows=4, N=50, K=100, group=64, experts=3, offsets=AT["offsets"], X=AT["a"], ldx=100, Wp=AT["q"], bias=AT["bias"], C=AT["c"], ldc=50, dtype=1, stream=None),
}
SIZES = [("ARG", dict(N=-1)), ("ARG", dict(K=-1)), ("SHAPE", dict(N=1 << 29, ldc=1 << 29, lddc=1 << 29)), ("SHAPE", dict(N=1 << 28, K=1 << 28, lda=1 << 28, ldc=1 << 28, lddc=1 << 28, ldx=1 << 28, ldw=1 << 28))]
EXPERTS = [("ARG", dict(experts=0)), ("SHAPE", dict(experts=1025))]
Q = 4 * 1 * (1024 + 128)  # bytes of an expert's 50 x 100 weights, groups of 64
BAD = {
    "lcma_gemm_experts": SIZES + EXPERTS + [("ARG", dict(b_layout=1)), ("ARG", dict(b_layout=3)), ("DTYPE", dict(dtype=3)), ("ARG", dict(rows=-1)), ("SHAPE", dict(rows=1 << 31))] +
                         [("ARG", {k: None}) for k in ("offsets", "A", "B", "C")] + [("ARG", dict(lda=99)), ("ARG", dict(ldc=49)), ("SHAPE", dict(lda=1 << 29)), ("SHAPE", dict(ldc=1 << 29)),
                          ("ARG", dict(A=AT["a"] + 1)), ("ARG", dict(B=AT["w"] + 1)), ("ARG", dict(C=AT["c"] + 1)), ("ARG", dict(offsets=AT["offsets"] + 2)), ("ARG", dict(C=AT["a"] + 798)),
                          ("ARG", dict(C=AT["w"] + 29998)), ("ARG", dict(C=AT["offsets"] + 14)), ("SHAPE", dict(rows=(1 << 31) - 1, N=1 << 24, ldc=1 << 24, A=1 << 60, C=1 << 61))],
    "lcma_gemm_experts_grad": SIZES + EXPERTS + [("DTYPE", dict(dtype=3)), ("ARG", dict(rows=-1)), ("SHAPE", dict(rows=1 << 31))] + [("ARG", {k: None}) for k in ("offsets", "dC", "A", "dW")] +
                              [("ARG", dict(lda=99)), ("ARG", dict(lddc=49)), ("SHAPE", dict(lda=1 << 29)), ("ARG", dict(dW=AT["a"] + 798)), ("ARG", dict(dW=AT["c"])), ("ARG", dict(dW=AT["offsets"] + 12)),
                               ("ARG", dict(dW=AT["w"] + 1)), ("SHAPE", dict(N=1 << 22, K=1 << 22, experts=1024, lda=1 << 22, lddc=1 << 22, dW=1 << 60))],
    "lcma_gated_silu": [("DTYPE", dict(dtype=9)), ("ARG", dict(rows=-1)), ("ARG", dict(F=-1)), ("SHAPE", dict(rows=1 << 31)), ("SHAPE", dict(F=1 << 26, ldx=1 << 27, ldy=1 << 26)), ("ARG", dict(X=None)),
                        ("ARG", dict(Y=None)), ("ARG", dict(ldx=99)), ("ARG", dict(ldy=49)), ("SHAPE", dict(ldx=1 << 29)), ("SHAPE", dict(ldy=1 << 29)), ("ARG", dict(X=AT["a"] + 1)),
                        ("ARG", dict(Y=AT["a"] + 798)), ("ARG", dict(Y=AT["a"]))],
    "lcma_gated_silu_grad": [("DTYPE", dict(dtype=-1)), ("ARG", dict(rows=-1)), ("ARG", dict(dY=None)), ("ARG", dict(X=None)), ("ARG", dict(dX=None)), ("ARG", dict(lddy=49)), ("ARG", dict(ldx=99)),
                             ("ARG", dict(lddx=99)), ("SHAPE", dict(lddy=1 << 29)), ("ARG", dict(dY=AT["dy"] + 1)), ("ARG", dict(dX=AT["a"])), ("ARG", dict(dX=AT["dy"] + 398))],
    "lcma_i4_quantize": SIZES + EXPERTS + [("DTYPE", dict(dtype=5)), ("ARG", dict(group=16)), ("ARG", dict(group=0)), ("ARG", dict(group=100)), ("ARG", dict(W=None)), ("ARG", dict(Wp=None)),
                                           ("ARG", dict(ldw=99)), ("SHAPE", dict(ldw=1 << 29)), ("ARG", dict(Wp=AT["q"] + 8)), ("ARG", dict(W=AT["w"] + 1)), ("ARG", dict(Wp=AT["w"] + 19984)),
                                           ("ARG", dict(W=AT["q"] + 2 * Q - 2))],
    "lcma_i4_prepare": SIZES + EXPERTS + [("ARG", dict(group=256)), ("ARG", dict(codes=None)), ("ARG", dict(scales=None)), ("ARG", dict(Wp=None)), ("ARG", dict(scales=AT["s"] + 2)),
                                          ("ARG", dict(Wp=AT["q"] + 4)), ("ARG", dict(codes=AT["q"] + 2 * Q - 1)), ("ARG", dict(scales=AT["q"]))],
    "lcma_i4_gemm_nt": SIZES + [("DTYPE", dict(dtype=3)), ("ARG", dict(M=-1)), ("SHAPE", dict(M=1 << 31)), ("ARG", dict(group=1)), ("ARG", dict(X=None)), ("ARG", dict(Wp=None)), ("ARG", dict(C=None)),
                                ("ARG", dict(ldx=99)), ("ARG", dict(ldc=49)), ("SHAPE", dict(ldx=1 << 29)), ("ARG", dict(X=AT["a"] + 1)), ("ARG", dict(C=AT["c"] + 1)), ("ARG", dict(Wp=AT["q"] + 8)),
                                ("ARG", dict(bias=AT["bias"] + 1)), ("ARG", dict(C=AT["q"] + Q - 2)), ("ARG", dict(C=AT["a"])), ("ARG", dict(C=AT["bias"] + 198)),
                                ("SHAPE", dict(M=(1 << 31) - 1, N=1 << 24, ldc=1 << 24, X=1 << 60, C=1 << 61))],
    "lcma_i4_gemm_experts": EXPERTS + [("ARG", dict(offsets=None)), ("ARG", dict(offsets=AT["offsets"] + 1)), ("ARG", dict(rows=-1)), ("ARG", dict(C=AT["q"] + 3 * Q - 2)),
                                       ("ARG", dict(C=AT["offsets"] + 14)), ("ARG", dict(C=AT["bias"] + 598)), ("ARG", dict(group=48))],
}


@pytest.mark.parametrize("name,status,change", [(n, s, c) for n, cases in BAD.items() for s, c in cases], ids=lambda v: str(v)[:40])
def test_refusals(B, name, status, change):
    args = {**CALLS[name], **{k: v for k, v in change.items() if k in CALLS[name]}}
    got = getattr(B.lib(), name)(*args.values())
    assert B.STATUS_NAMES[got] == "ERR_" + status
    assert B.lib().lcma_last_error().decode().startswith(name + ":")


@pytest.mark.parametrize("name,change", [("lcma_gemm_experts", dict(rows=0, offsets=None, A=None, B=None, C=None)), ("lcma_gemm_experts", dict(N=0, C=None, B=None)),
                                         ("lcma_gemm_experts_grad", dict(N=0, dW=None)), ("lcma_gemm_experts_grad", dict(K=0, dW=None)), ("lcma_gated_silu", dict(rows=0, X=None, Y=None)),
                                         ("lcma_gated_silu", dict(F=0, X=None, Y=None)), ("lcma_gated_silu_grad", dict(rows=0, X=None, dY=None, dX=None)), ("lcma_i4_quantize", dict(N=0, W=None, Wp=None)),
                                         ("lcma_i4_prepare", dict(K=0, codes=None, scales=None, Wp=None)), ("lcma_i4_gemm_nt", dict(M=0, X=None, C=None)), ("lcma_i4_gemm_nt", dict(N=0, C=None)),
                                         ("lcma_i4_gemm_experts", dict(rows=0, offsets=None, X=None, C=None))], ids=lambda v: str(v)[:40])
def test_nothing_to_do_is_no_error(B, name, change):
    assert getattr(B.lib(), name)(*{**CALLS[name], **change}.values()) == B.LCMA_OK


def test_sizes(B):
    size = B.lcma_i4_prepared_bytes
    assert [size(n, k, g) for n, k, g in ((0, 5, 32), (5, 0, 64), (1, 1, 128), (16, 128, 32), (17, 128, 64), (50, 100, 64))] == [0, 0, 1088, 1280, 2304, Q]
    assert size(14336, 4096, 128) == 14336 * (4096 // 2 + 4096 // 128 * 4)
    assert size(-1, 8, 32) == size(8, -1, 32) == size(8, 8, 16) == size(1 << 29, 1, 32) == size(1 << 28, 1 << 28, 32) == -1


def test_the_binding_names_the_argument_it_refuses(B):
    import torch
    calls = B._native()
    x, w, o = torch.zeros((4, 8)), torch.zeros((2, 4, 8)), torch.zeros(3, dtype=torch.int32)
    for f, args, what in [(calls.gemm_experts, (x, o, w, x, True), "A: expected a tensor on the GPU"), (calls.gemm_experts, (x, o, x, x, True), "W: expected three dimensions"),
                          (calls.gemm_experts_grad, (x, x, o, w), "A: expected a tensor on the GPU"), (calls.gated_silu, (torch.zeros((4, 7)), x), "X: expected rows x 2 F"),
                          (calls.gated_silu_grad, (x, x, x), "X: expected a tensor on the GPU"), (calls.i4_quantize, (torch.zeros(4), 32, x), "W: expected two or three dimensions"),
                          (calls.i4_gemm_nt, (x, x, 7, 32, None), "C: expected a tensor"), (calls.i4_gemm_experts, (x, o[:1], x, x, 32, None), "offsets: expected experts")]:
        with pytest.raises(AssertionError, match=what):
            f(*args)
    with pytest.raises(TypeError):
        calls.gated_silu(x)
    with pytest.raises(TypeError):
        calls.i4_quantize(w, "many", x)
