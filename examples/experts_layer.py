"""A mixture-of-experts feed-forward layer: served in 8-bit integers or with 4-bit weights, and trained in bf16.

  python examples/experts_layer.py [--tokens 4096] [--experts 8] [--top 2] [--hidden 2048] [--ffn 4096]

Serving: the tokens are sorted by expert, quantised on their way into the experts' order, multiplied with all experts' gate and up weights in one call,
gated and quantised again, multiplied with the down weights, and summed back into tokens with the router's weights.  Nothing leaves the GPU and
the host never learns how many rows an expert has.

For single tokens the weights may have 4 bits, with a scale for each group of columns; the activations stay in 16.

Training: the movement, the products over all experts, the gate between them and the gradients of all these are the library's calls as well.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_06057_amd import binding as lcma  # noqa: E402


def route(x, router, top):
    """Expert numbers (tokens x top, int32) and weights (fp32, they sum to one) of a linear router."""
    best, ids = (x.float() @ router.float().t()).topk(top, dim=1)
    return ids.int(), torch.softmax(best, dim=1)


class ServedExperts:
    """Experts with 8-bit weights: w_in (experts x 2 ffn x hidden: gate rows, then up rows) and w_out (experts x hidden x ffn)."""

    def __init__(self, w_in, w_out):
        self.experts, self.hidden, self.ffn = w_in.shape[0], w_in.shape[2], w_out.shape[2]

        def quantised(w):  # a channel is a row: all experts at once
            q, s = lcma.lcma_i8_quantize(w.reshape(-1, w.shape[2]))
            return q.view(w.shape[0], w.shape[1], -1), s.view(w.shape[0], w.shape[1])

        self.q_in, self.s_in = quantised(w_in)
        self.q_out, self.s_out = quantised(w_out)

    def __call__(self, x, ids, weights):
        rows = ids.numel()
        _, position, offsets = lcma.lcma_tokens_sort(ids, self.experts)
        q, s = lcma.lcma_i8_quantize_dispatch(x, position)
        h = lcma.lcma_i8_gemm_experts(q, s, offsets, self.q_in, self.s_in, x.new_empty((rows, 2 * self.ffn)), self.hidden)
        q, s = lcma.lcma_i8_quantize(h, gated=True)
        y = lcma.lcma_i8_gemm_experts(q, s, offsets, self.q_out, self.s_out, x.new_empty((rows, self.hidden)), self.ffn)
        return lcma.lcma_tokens_combine(y, position, weights)


class ServedExperts4:
    """Experts whose weights have 4 bits and a scale for each `group` of columns, laid out as ServedExperts': for the few rows of single tokens, which stay in 16 bits."""

    def __init__(self, w_in, w_out, group=128):
        self.experts, self.ffn, self.hidden, self.group = w_in.shape[0], w_in.shape[1] // 2, w_in.shape[2], group
        self.q_in, self.q_out = lcma.lcma_i4_quantize(w_in, group), lcma.lcma_i4_quantize(w_out, group)

    def __call__(self, x, ids, weights):
        rows = ids.numel()
        _, position, offsets = lcma.lcma_tokens_sort(ids, self.experts)
        h = lcma.lcma_i4_gemm_experts(lcma.lcma_tokens_dispatch(x, position), offsets, self.q_in, x.new_empty((rows, 2 * self.ffn)), self.group)
        y = lcma.lcma_i4_gemm_experts(lcma.lcma_gated_silu(h), offsets, self.q_out, x.new_empty((rows, self.hidden)), self.group)
        return lcma.lcma_tokens_combine(y, position, weights)


def asked_for(ctx, n):
    """Which of the n inputs' gradients a backward pass has to give: those that autograd names, all where it is called by itself.
    The library's calls have no derivatives of their own: with create_graph, where gradients are computed to be differentiated, they would count as constants."""
    needs = getattr(ctx, "needs_input_grad", None)
    if needs is not None and torch.is_grad_enabled():
        raise RuntimeError("the experts' layer has no second derivative: create_graph is not supported")
    return needs or (True,) * n


class TrainedLinearExperts(torch.autograd.Function):
    """y[t] = sum over j of weights[t, j] * W[ids[t, j]] x[t], with the gradients of x, of the experts' matrices W (experts x out x in) and of weights."""

    @staticmethod
    def forward(ctx, x, w, ids, weights):
        _, position, offsets = lcma.lcma_tokens_sort(ids, w.shape[0])
        rows = lcma.lcma_tokens_dispatch(x, position)
        y = lcma.lcma_gemm_experts(rows, offsets, w)
        ctx.save_for_backward(rows, w, position, offsets, weights, y)
        return lcma.lcma_tokens_combine(y, position, weights)

    @staticmethod
    def backward(ctx, grad):
        need_x, need_w, _, need_weights = asked_for(ctx, 4)
        rows, w, position, offsets, weights, y = ctx.saved_tensors
        dy, dweights = lcma.lcma_tokens_combine_grad(grad.contiguous(), y, position, weights)
        dx = lcma.lcma_tokens_combine(lcma.lcma_gemm_experts(dy, offsets, w, b_nk=False), position) if need_x else None
        return dx, lcma.lcma_gemm_experts_grad(dy, rows, offsets) if need_w else None, None, dweights if need_weights else None


class TrainedExperts(torch.autograd.Function):
    """The whole layer: y[t] = sum over j of weights[t, j] * w_out[e] (silu(g) * u), (g, u) = w_in[e] x[t], e = ids[t, j], with the gradients of x, of both of the experts' matrices
    (w_in: experts x 2 ffn x hidden, gate rows first; w_out: experts x hidden x ffn) and of weights.  What the gate gives is computed anew for the gradients instead of kept."""

    @staticmethod
    def forward(ctx, x, w_in, w_out, ids, weights):
        _, position, offsets = lcma.lcma_tokens_sort(ids, w_in.shape[0])
        rows = lcma.lcma_tokens_dispatch(x, position)
        h = lcma.lcma_gemm_experts(rows, offsets, w_in)
        y = lcma.lcma_gemm_experts(lcma.lcma_gated_silu(h), offsets, w_out)
        ctx.save_for_backward(rows, h, y, w_in, w_out, position, offsets, weights)
        return lcma.lcma_tokens_combine(y, position, weights)

    @staticmethod
    def backward(ctx, grad):
        need_x, need_in, need_out, _, need_weights = asked_for(ctx, 5)
        rows, h, y, w_in, w_out, position, offsets, weights = ctx.saved_tensors
        dy, dweights = lcma.lcma_tokens_combine_grad(grad.contiguous(), y, position, weights)
        dx = dw_in = dw_out = None
        if need_out:
            dw_out = lcma.lcma_gemm_experts_grad(dy, lcma.lcma_gated_silu(h), offsets)
        if need_x or need_in:
            dh = lcma.lcma_gated_silu_grad(lcma.lcma_gemm_experts(dy, offsets, w_out, b_nk=False), h)
            dx = lcma.lcma_tokens_combine(lcma.lcma_gemm_experts(dh, offsets, w_in, b_nk=False), position) if need_x else None
            dw_in = lcma.lcma_gemm_experts_grad(dh, rows, offsets) if need_in else None
        return dx, dw_in, dw_out, None, dweights if need_weights else None


def train(x, target, w, router, top, steps):
    """Gradient descent on copies of the experts' matrices (in the type of x, updated in fp32) and of the router, for tokens x of independent N(0, 1); the loss
    of every step."""
    master, router, losses = w.float().clone(), router.clone(), []
    rate = 0.5 / (1 + (x.shape[1] / x.shape[0]) ** 0.5) ** 2  # half of what the largest eigenvalue of x^T x / tokens allows
    for _ in range(steps):
        wb, r = master.to(x.dtype, copy=True).requires_grad_(), router.clone().requires_grad_()
        ids, weights = route(x, r, top)
        out = TrainedLinearExperts.apply(x, wb, ids, weights)
        loss = 0.5 * (out.float() - target.float()).square().sum(dim=1).mean()
        loss.backward()
        master -= rate * wb.grad.float()
        router -= rate / w.shape[1] * r.grad  # (its gradient adds up all columns of the result)
        losses.append(loss.item())
    return losses


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("tokens", 4096), ("experts", 8), ("top", 2), ("hidden", 2048), ("ffn", 4096)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    gen = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *shape, spread=1.0: (torch.randn(shape, device="cuda", generator=gen) * spread).bfloat16()
    x, router = normal(a.tokens, a.hidden), torch.randn((a.experts, a.hidden), device="cuda", generator=gen) / a.hidden ** 0.5
    w_in, w_out = normal(a.experts, 2 * a.ffn, a.hidden, spread=0.02), normal(a.experts, a.hidden, a.ffn, spread=0.02)
    ids, weights = route(x, router, a.top)

    layer = ServedExperts(w_in, w_out)
    got = layer(x, ids, weights).float()
    want = torch.zeros_like(got)
    for e in range(a.experts):
        t, j = (ids == e).nonzero(as_tuple=True)
        g, u = (x[t].float() @ w_in[e].float().t()).chunk(2, dim=1)
        want.index_add_(0, t, weights[t, j, None] * ((torch.nn.functional.silu(g) * u) @ w_out[e].float().t()))
    print(f"served in 8 bit: relative error against the unquantised layer {((got - want).norm() / want.norm()).item():.4f}")
    four = ServedExperts4(w_in, w_out)
    print(f"served in 4 bit: {((four(x, ids, weights).float() - want).norm() / want.norm()).item():.4f}")

    def timed(f):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        for _ in range(3):
            f()
        begin.record()
        for _ in range(20):
            f()
        end.record()
        torch.cuda.synchronize()
        return begin.elapsed_time(end) / 20

    ms = timed(lambda: layer(x, ids, weights))
    ops = 2.0 * ids.numel() * 3 * a.ffn * a.hidden
    print(f"{a.tokens} tokens, {a.top} of {a.experts} experts, {a.hidden} x {a.ffn}: {ms * 1e3:.0f} us, {ops / ms / 1e9:.0f} TOP/s")
    one = [t[:1].contiguous() for t in (x, ids, weights)]
    print(f"one token: 8 bit {timed(lambda: layer(*one)) * 1e3:.0f} us, 4 bit {timed(lambda: four(*one)) * 1e3:.0f} us")
    leaves = [t.clone().requires_grad_() for t in (x, w_in, w_out, weights)]
    ms = timed(lambda: TrainedExperts.apply(*leaves[:3], ids, leaves[3]).backward(x))
    print(f"a training step of the layer, forward and back: {ms * 1e3:.0f} us, {3 * ops / ms / 1e9:.0f} TFLOP/s")

    w = normal(a.experts, 512, a.hidden, spread=a.hidden ** -0.5)
    losses = train(x, normal(a.tokens, 512, spread=0.1), w, router, a.top, 8)
    print("training, loss of every step: " + " ".join(f"{v:.4f}" for v in losses))


if __name__ == "__main__":
    main()
