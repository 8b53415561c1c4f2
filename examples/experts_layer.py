"""A mixture-of-experts feed-forward layer: served in 8-bit integers, and trained in bf16.

  python examples/experts_layer.py [--tokens 4096] [--experts 8] [--top 2] [--hidden 2048] [--ffn 4096]

Serving: the tokens are sorted by expert, quantised on their way into the experts' order, multiplied with all experts' gate and up weights in one call,
gated and quantised again, multiplied with the down weights, and summed back into tokens with the router's weights.  Nothing leaves the GPU and
the host never learns how many rows an expert has.

Training: the movement and its gradients are the library's calls as well; the products of each expert are its 16-bit ones.
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


def _product(a, b, b_nk):
    """a b (a b^T) by the library's plain product, whose sizes along both axes of b are multiples of 8."""
    c = a.new_empty((a.shape[0], b.shape[0] if b_nk else b.shape[1]))
    return lcma.lcma_gemm_nt(a, b, c) if b_nk else lcma.lcma_gemm(a, b, c)


def _padded(t):
    """t with zero rows behind, to a multiple of 8."""
    return torch.nn.functional.pad(t, (0, 0, 0, -t.shape[0] % 8))


class TrainedLinearExperts(torch.autograd.Function):
    """y[t] = sum over j of weights[t, j] * W[ids[t, j]] x[t], with the gradients of x, of the experts' matrices W (experts x out x in) and of weights."""

    @staticmethod
    def forward(ctx, x, w, ids, weights):
        _, position, offsets = lcma.lcma_tokens_sort(ids, w.shape[0])
        rows = lcma.lcma_tokens_dispatch(x, position)
        ends = offsets.tolist()  # (the products of the experts are calls of their own: the host needs their sizes)
        y = torch.zeros((rows.shape[0], w.shape[1]), dtype=x.dtype, device=x.device)
        for e, (a, b) in enumerate(zip(ends, ends[1:])):
            if b > a:
                y[a:b] = _product(rows[a:b], w[e], True)
        ctx.save_for_backward(rows, w, position, weights, y)
        ctx.ends = ends
        return lcma.lcma_tokens_combine(y, position, weights)

    @staticmethod
    def backward(ctx, grad):
        rows, w, position, weights, y = ctx.saved_tensors
        dy, dweights = lcma.lcma_tokens_combine_grad(grad.contiguous(), y, position, weights)
        drows, dw = torch.zeros_like(rows), torch.zeros_like(w)
        for e, (a, b) in enumerate(zip(ctx.ends, ctx.ends[1:])):
            if b > a:
                drows[a:b] = _product(dy[a:b], w[e], False)
                dw[e] = _product(_padded(dy[a:b]).t().contiguous(), _padded(rows[a:b]), False)
        return lcma.lcma_tokens_combine(drows, position), dw, None, dweights


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
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for _ in range(3):
        layer(x, ids, weights)
    begin.record()
    for _ in range(20):
        layer(x, ids, weights)
    end.record()
    torch.cuda.synchronize()
    ms = begin.elapsed_time(end) / 20
    ops = 2.0 * ids.numel() * 3 * a.ffn * a.hidden
    print(f"{a.tokens} tokens, {a.top} of {a.experts} experts, {a.hidden} x {a.ffn}: {ms * 1e3:.0f} us, {ops / ms / 1e9:.0f} TOP/s")

    w = normal(a.experts, 512, a.hidden, spread=a.hidden ** -0.5)
    losses = train(x, normal(a.tokens, 512, spread=0.1), w, router, a.top, 8)
    print("training, loss of every step: " + " ".join(f"{v:.4f}" for v in losses))


if __name__ == "__main__":
    main()
