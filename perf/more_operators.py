"""A mixture-of-experts layer's products in its own type, with both gradients; its gate with its gradient; linear layers whose weights are 4-bit integers
with a scale for each group, alone and over experts: timed and checked cases.

A case is one pass of one kind:

  product   rows in expert order, each expert's times its weights (experts x N x K)
  grads     the two gradients of such a product: of the rows, and of every expert's weights
  gated     silu(gate) * up of every row, and its gradient
  linear4   activations times N x K weights of 4 bits, a scale for each group of 32, 64 or 128 along K
  experts4  the same over experts

Where `own` is false a pass is elementary torch in 32 bits; where it is true, the calls that a user makes of the library.
"""
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _experts(kind, dtype, T, top, E, N, K, drop=0.0, group=0):
    """T tokens with `top` of E experts each, N columns, K summed; drop: share of slots without an expert, whose rows are behind all others."""
    return {"kind": kind, "dtype": dtype, "T": T, "top": top, "E": E, "N": N, "K": K, "drop": drop, "group": group}


def _gated(dtype, T, F, pad=0):
    return {"kind": "gated", "dtype": dtype, "T": T, "F": F, "pad": pad}


def _linear4(dtype, M, N, K, group, bias=False, pad=0):
    return {"kind": "linear4", "dtype": dtype, "M": M, "N": N, "K": K, "group": group, "bias": bias, "pad": pad}


def listed():
    cases = [
        # a single token, two of eight experts: their weights are read once for it
        ("product_bf16_1x2of8_28672x4096", _experts("product", "bf16", 1, 2, 8, 28672, 4096)),
        # a short prompt over many small experts, about a hundred rows for each, padding tokens, columns off the vectors
        ("product_f16_1021x6of64_2815x2056", _experts("product", "f16", 1021, 6, 64, 2815, 2056, 0.05)),
        # a training step's tokens through the first product of large experts
        ("product_bf16_8192x2of8_28672x4096", _experts("product", "bf16", 8192, 2, 8, 28672, 4096)),
        # a small batch trained: most experts get a few rows
        ("grads_bf16_16x2of8_2048x1024", _experts("grads", "bf16", 16, 2, 8, 2048, 1024)),
        # fp32, every size odd, padding tokens
        ("grads_f32_777x3of12_1001x515", _experts("grads", "f32", 777, 3, 12, 1001, 515, 0.1)),
        # a training step's tokens through the second product
        ("grads_bf16_8192x2of8_4096x14336", _experts("grads", "bf16", 8192, 2, 8, 4096, 14336)),
        # the gate of a token's two experts
        ("gated_bf16_2x14336", _gated("bf16", 2, 14336)),
        # of a training step's rows
        ("gated_bf16_16384x14336", _gated("bf16", 16384, 14336)),
        # a single token through a linear layer
        ("linear4_bf16_1x14336x4096_g128", _linear4("bf16", 1, 14336, 4096, 128)),
        # a few sequences, every size off the vectors, rows of a wider tensor, a bias, small groups
        ("linear4_f16_45x1001x1545_g32", _linear4("f16", 45, 1001, 1545, 32, True, 24)),
        # single tokens of eight sequences, large experts
        ("experts4_bf16_8x2of8_28672x4096_g128", _experts("experts4", "bf16", 8, 2, 8, 28672, 4096, 0.0, 128)),
        # a batch of sequences over many small experts, a few rows for each
        ("experts4_f16_61x6of64_2816x2048_g64", _experts("experts4", "f16", 61, 6, 64, 2816, 2048, 0.05, 64)),
    ]
    return [dict(c, name=n) for n, c in cases]


def _size(rng, lo, hi):
    """A size spread evenly over the logarithm of [lo, hi]; a whole multiple of 64 as often as not, where it is large enough."""
    v = max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))
    return v // 64 * 64 if v >= 128 and rng.random() < 0.5 else v


def draw(rng):
    kind = rng.choice(["product", "product", "grads", "grads", "gated", "linear4", "linear4", "experts4"])
    while True:
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        if kind == "gated":
            c = _gated(dtype, _size(rng, 1, 16384), _size(rng, 64, 14336), rng.choice([0, 0, 8, 5]))
            if c["T"] * c["F"] * (2 if dtype == "f32" else 1) <= 16384 * 14336:
                return c
            continue
        if kind == "linear4":
            c = _linear4(dtype, _size(rng, 1, 256), _size(rng, 64, 28672), _size(rng, 64, 14336), rng.choice([32, 64, 128]), rng.random() < 0.5, rng.choice([0, 0, 8, 24, 5]))
            if c["N"] * c["K"] <= 14336 * 8192:
                return c
            continue
        T = _size(rng, 1, 64 if kind == "experts4" else 8192)
        c = _experts(kind, dtype, T, rng.choice([1, 2, 4, 6, 8]), rng.choice([8, 16, 60, 64, 128]), _size(rng, 64, 28672), _size(rng, 64, 14336),
                     rng.choice([0.0, 0.0, 0.1]), rng.choice([32, 64, 128]) if kind == "experts4" else 0)
        weights, rows = c["E"] * c["N"] * c["K"] * (2 if dtype == "f32" else 1), T * c["top"]
        # (fp32 products run at a sixteenth of the rate)
        if weights <= 8 * 4096 * 28672 and rows * c["N"] * c["K"] * (8 if dtype == "f32" else 1) * (2 if kind == "grads" else 1) <= 8192 * 2 * 4096 * 28672:
            return c


# ------------------------------------------------------------------ what a program has in hand
def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _normal(gen, shape, dtype, spread=1.0):
    return torch.empty(shape, device="cuda", dtype=torch.float32).normal_(0.0, spread, generator=gen).to(dtype)


def _empty(shape, dtype):
    return torch.empty(shape, device="cuda", dtype=dtype)


def _offsets(gen, case):
    """First row of every expert, as a router and a sort leave them: some experts are more popular than others, rows of dropped slots are behind."""
    T, top, E = case["T"], case["top"], case["E"]
    logits = torch.randn((T, E), device="cuda", generator=gen) + 0.5 * torch.randn((E,), device="cuda", generator=gen)
    ids = logits.topk(top, dim=1).indices.reshape(-1)
    kept = torch.rand((T * top,), device="cuda", generator=gen) >= case["drop"]
    count = torch.zeros((E,), device="cuda", dtype=torch.int64).index_add_(0, ids, kept.long())
    return torch.cat([torch.zeros((1,), device="cuda", dtype=torch.int64), count.cumsum(0)]).int()


def _weights4(gen, lead, N, K, group):
    """4-bit codes (-8 .. 7, a byte each) and the scale of each group, as a quantised weight matrix has them."""
    codes = torch.empty((*lead, N, K), device="cuda", dtype=torch.float16).normal_(0.0, 3.0, generator=gen).round_().clamp_(-8, 7).to(torch.int8)
    scales = torch.empty((*lead, N, (K + group - 1) // group), device="cuda").uniform_(0.7, 1.3, generator=gen) * (0.02 / 3)
    return codes, scales


def _inputs(case, seed):
    gen, dt, kind = _generator(seed), DTYPES[case["dtype"]], case["kind"]
    st = {"kind": kind}
    if kind == "gated":
        T, F, pad = case["T"], case["F"], case["pad"]
        st["x"] = _normal(gen, (T, 2 * F + pad), dt, 1.5)[:, : 2 * F]
        st["dy"] = _normal(gen, (T, F + pad), dt)[:, :F]
        st["y"], st["dx"] = _empty((T, F), dt), _empty((T, 2 * F), dt)
        return st
    N, K, group = case["N"], case["K"], case["group"]
    if kind == "linear4":
        M, lead = case["M"], ()
        st["x"] = _normal(gen, (M, K + case["pad"]), dt)[:, :K]
        st["bias"] = _normal(gen, (N,), torch.float32) if case["bias"] else None
    else:
        M, lead = case["T"] * case["top"], (case["E"],)
        st["offsets"] = _offsets(gen, case)
        st["x"] = _normal(gen, (M, K), dt)
    st["group"] = group
    if group:
        st["codes"], st["scales"] = _weights4(gen, lead, N, K, group)
    else:
        st["w"] = _normal(gen, (*lead, N, K), dt, 0.02)
    if kind == "grads":
        st["dc"] = _normal(gen, (M, N), dt)
        st["dx"], st["dw"] = _empty((M, K), dt), _empty((*lead, N, K), dt)
    else:
        st["c"] = _empty((M, N), dt)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own and st.get("group"):  # (the library lays 4-bit weights out once)
        from paper_2605_06057_amd import binding as lib

        st["w"] = lib.lcma_i4_prepare(st["codes"], st["scales"], st["group"])
    return st


# ------------------------------------------------------------------ plain forms
def _blocks(rows, offsets, most, at):
    """Each expert's rows in a block of its own, `most` rows with zeros behind."""
    E = offsets.numel() - 1
    out = torch.zeros((E * most + 1, rows.shape[1]), device=rows.device)
    out[at] = torch.where((at < E * most)[:, None], rows, torch.zeros((), device=rows.device))
    return out[:-1].view(E, most, -1)


def _places(offsets, n):
    """How many rows the largest expert has, and the place of every row among the blocks (the last one: rows of no expert)."""
    E = offsets.numel() - 1
    row = torch.arange(n, device=offsets.device)
    e = (row[:, None] >= offsets[None, 1:]).sum(1)
    most = max(1, int((offsets[1:] - offsets[:-1]).max()))
    return most, torch.where(e < E, e * most + row - offsets[e.clamp(max=E)], torch.full_like(row, E * most))


def _rows(blocks, at):
    E, most, N = blocks.shape
    return torch.cat([blocks.reshape(E * most, N), torch.zeros((1, N), device=blocks.device)])[at]


def _dequantised(st, K):
    return st["codes"].float() * st["scales"].repeat_interleave(st["group"], dim=-1)[..., :K]


def _plain(st):
    kind, x = st["kind"], st["x"]
    if kind == "gated":
        (g, u), dy = x.float().chunk(2, dim=1), st["dy"].float()
        s = 1 / (1 + torch.exp(-g))
        return {"y": (g * s * u).to(x.dtype), "dx": torch.cat([dy * u * s * (1 + g * (1 - s)), dy * g * s], dim=1).to(x.dtype)}
    w = _dequantised(st, x.shape[1]) if st["group"] else st["w"].float()
    if kind == "linear4":
        c = x.float() @ w.t()
        return {"c": (c if st["bias"] is None else c + st["bias"]).to(x.dtype)}
    offsets = st["offsets"].long()
    most, at = _places(offsets, x.shape[0])
    blocks = _blocks(x.float(), offsets, most, at)
    if kind != "grads":
        return {"c": _rows(torch.bmm(blocks, w.transpose(1, 2)), at).to(x.dtype)}
    dc = _blocks(st["dc"].float(), offsets, most, at)
    return {"dx": _rows(torch.bmm(dc, w), at).to(x.dtype), "dw": torch.bmm(dc.transpose(1, 2), blocks).to(x.dtype)}


# ------------------------------------------------------------------ a pass
def run(st):
    if not own:
        return _plain(st)
    from paper_2605_06057_amd import binding as lib

    kind, x = st["kind"], st["x"]
    if kind == "gated":
        return {"y": lib.lcma_gated_silu(x, st["y"]), "dx": lib.lcma_gated_silu_grad(st["dy"], x, st["dx"])}
    if kind == "linear4":
        return {"c": lib.lcma_i4_gemm_nt(x, st["w"], st["c"], st["group"], st["bias"])}
    if kind == "experts4":
        return {"c": lib.lcma_i4_gemm_experts(x, st["offsets"], st["w"], st["c"], st["group"])}
    if kind == "product":
        return {"c": lib.lcma_gemm_experts(x, st["offsets"], st["w"], st["c"])}
    return {"dx": lib.lcma_gemm_experts(st["dc"], st["offsets"], st["w"], st["dx"], b_nk=False),
            "dw": lib.lcma_gemm_experts_grad(st["dc"], x, st["offsets"], st["dw"])}


# ------------------------------------------------------------------ what it cannot do without
def work(case):
    es, kind = 4 if case["dtype"] == "f32" else 2, case["kind"]
    if kind == "gated":
        # the rows, their gates' values, the gradient of those, the gradient of the rows (a pass forward and a pass back, each reads the rows)
        return {"bytes": case["T"] * case["F"] * es * 8, "flops": 20.0 * case["T"] * case["F"]}
    N, K = case["N"], case["K"]
    weight = K / 2 + 4 * ((K + case["group"] - 1) // case["group"]) if case["group"] else K * es  # bytes of a row of weights
    if kind == "linear4":
        M = case["M"]
        return {"bytes": (M * K + M * N) * es + N * weight + 4 * N * case["bias"], "flops": 2.0 * M * N * K}
    T, top, E = case["T"], case["top"], case["E"]
    n, kept = T * top, T * top * (1 - case["drop"])
    hit = E * (1 - (1 - top / E * (1 - case["drop"])) ** T)  # experts that some token goes to, were they equally popular
    if kind == "grads":
        # both products read the gradient; the weights' gradient is written for all experts
        return {"bytes": (2 * n * N + 2 * n * K) * es + (hit + E) * N * weight, "flops": 4.0 * kept * N * K}
    return {"bytes": n * (K + N) * es + hit * N * weight, "flops": 2.0 * kept * N * K}


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    st = _inputs(case, seed)
    x = st["x"].double()
    if case["kind"] == "gated":
        F = case["F"]
        g, u, dy = x[:, :F], x[:, F:], st["dy"].double()
        s = torch.sigmoid(g)
        return {"y": u * g * s, "dx": torch.cat([dy * u * (s + g * s * (1 - s)), dy * (g * s)], dim=1)}

    def weights(e):
        if not case["group"]:
            return st["w"][e].double()
        codes, scales = (st["codes"], st["scales"]) if e is None else (st["codes"][e], st["scales"][e])
        k = torch.arange(case["K"], device="cuda")
        return codes.double() * scales.double()[:, k // case["group"]]

    if case["kind"] == "linear4":
        c = x @ weights(None).t()
        return {"c": c if st["bias"] is None else c + st["bias"].double()}
    ends = st["offsets"].tolist()
    n, N, K, E = x.shape[0], case["N"], case["K"], case["E"]
    zeros = lambda *shape: torch.zeros(shape, device="cuda", dtype=torch.float64)
    if case["kind"] == "grads":
        dc, dx, dw = st["dc"].double(), zeros(n, K), zeros(E, N, K)
        for e in range(E):
            a, b = ends[e], ends[e + 1]
            if b > a:
                dx[a:b] = dc[a:b] @ weights(e)
                dw[e] = dc[a:b].t() @ x[a:b]
        return {"dx": dx, "dw": dw}
    c = zeros(n, N)
    for e in range(E):
        a, b = ends[e], ends[e + 1]
        if b > a:
            c[a:b] = x[a:b] @ weights(e).t()
    return {"c": c}
