"""The 8-bit-integer linear layer, the same over experts, and the tokens' way to their experts and back: timed and checked cases.

A case is one pass of one kind:

  linear   activations quantised to 8 bits with a scale for each token, times N x K weights held in 8 bits with a scale for each channel
  route    a training step's movement of tokens: sort by expert, dispatch, combine with the router's weights, and the gradients of both
  up       the first product of an experts' layer in 8 bits: sort, quantise into the experts' order, one product over all experts
  down     the second: gated SiLU quantised, one product over all experts, the rows combined into tokens with the router's weights

Where `own` is false a pass is elementary torch in 32 bits; where it is true, the calls that a user makes of the library.
"""
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _linear(dtype, M, N, K, bias=False, pad=0):
    return {"kind": "linear", "dtype": dtype, "M": M, "N": N, "K": K, "bias": bias, "pad": pad}


def _experts(kind, dtype, T, top, E, H, F, drop=0.0):
    """T tokens of H values, `top` of E experts each, F columns of a product (route: none); drop: share of slots without an expert."""
    return {"kind": kind, "dtype": dtype, "T": T, "top": top, "E": E, "H": H, "F": F, "drop": drop}


def listed():
    cases = [
        # a single token through a linear layer: the weights are read once for it
        ("linear_bf16_1x14336x4096", _linear("bf16", 1, 14336, 4096)),
        # a few sequences, every size off the vectors, rows of a wider tensor, a bias
        ("linear_f16_45x1001x1545", _linear("f16", 45, 1001, 1545, True, 24)),
        # a short prompt, results kept in fp32
        ("linear_f32_333x4096x4096", _linear("f32", 333, 4096, 4096)),
        # a prompt through the feed-forward layer's first product
        ("linear_bf16_8192x14336x4096", _linear("bf16", 8192, 14336, 4096)),
        # a small batch on its way to two of eight experts
        ("route_bf16_16x2of8x4096", _experts("route", "bf16", 16, 2, 8, 4096, 0)),
        # many small experts, padding tokens without an expert, odd sizes, gradients in fp32
        ("route_f32_4099x6of60x1543", _experts("route", "f32", 4099, 6, 60, 1543, 0, 0.1)),
        # a training step's tokens
        ("route_bf16_16384x4of64x4096", _experts("route", "bf16", 16384, 4, 64, 4096, 0)),
        # single tokens of eight sequences: most experts are hit, each by a few rows
        ("up_bf16_8x2of8x4096x28672", _experts("up", "bf16", 8, 2, 8, 4096, 28672)),
        # a short prompt over many small experts: about a hundred rows for each
        ("up_f16_1021x6of64x2048x2816", _experts("up", "f16", 1021, 6, 64, 2048, 2816, 0.05)),
        # a prompt, large experts
        ("up_bf16_8192x2of8x4096x28672", _experts("up", "bf16", 8192, 2, 8, 4096, 28672)),
        # the second product for one token
        ("down_bf16_1x2of8x4096x14336", _experts("down", "bf16", 1, 2, 8, 4096, 14336)),
        # the second product for a prompt
        ("down_bf16_4096x2of8x4096x14336", _experts("down", "bf16", 4096, 2, 8, 4096, 14336)),
    ]
    return [dict(c, name=n) for n, c in cases]


def _size(rng, lo, hi):
    """A size spread evenly over the logarithm of [lo, hi]; a whole multiple of 64 as often as not, where it is large enough."""
    v = max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))
    return v // 64 * 64 if v >= 128 and rng.random() < 0.5 else v


def draw(rng):
    kind = rng.choice(["linear", "linear", "route", "up", "down"])
    while True:
        if kind == "linear":
            c = _linear(rng.choice(["bf16", "bf16", "f16", "f32"]), _size(rng, 1, 8192), _size(rng, 64, 14336), _size(rng, 64, 14336),
                        rng.random() < 0.5, rng.choice([0, 0, 8, 24, 5]))
            if c["M"] * c["N"] * c["K"] <= 8192 * 14336 * 4096:
                return c
            continue
        top = rng.choice([1, 2, 4, 6, 8])
        E = rng.choice([8, 16, 60, 64, 128])
        drop = rng.choice([0.0, 0.0, 0.1])
        if kind == "route":
            c = _experts(kind, rng.choice(["bf16", "f16", "f32"]), _size(rng, 1, 16384), top, E, _size(rng, 64, 8192), 0, drop)
            if c["T"] * top * c["H"] * (2 if c["dtype"] == "f32" else 1) <= 16384 * 4 * 4096:
                return c
            continue
        c = _experts(kind, rng.choice(["bf16", "bf16", "f16"]), _size(rng, 1, 8192), top, E, _size(rng, 256, 4096), _size(rng, 128, 28672 if kind == "up" else 14336), drop)
        if E * c["H"] * c["F"] <= 8 * 4096 * 28672 and c["T"] * top * c["H"] * c["F"] <= 8192 * 2 * 4096 * 14336:
            return c


# ------------------------------------------------------------------ what a program has in hand
def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _normal(gen, shape, dtype, spread=1.0):
    return torch.empty(shape, device="cuda", dtype=torch.float32).normal_(0.0, spread, generator=gen).to(dtype)


def _weights(gen, lead, N, K):
    """8-bit codes as a quantised weight matrix has them, rows padded with zeros to whole 128 bytes, and a scale for each row."""
    codes = torch.zeros((*lead, N, (K + 127) // 128 * 128), device="cuda", dtype=torch.int8)
    codes[..., :K] = torch.empty((*lead, N, K), device="cuda").normal_(0.0, 127.0 / 4, generator=gen).round_().clamp_(-127, 127)
    scales = torch.empty((*lead, N), device="cuda").uniform_(0.8, 1.2, generator=gen) * (4 * 0.02 / 127)
    return codes, scales


def _router(gen, case):
    """Expert numbers (some experts more popular than others, -1: none) and the softmax weights of the chosen ones."""
    T, top, E = case["T"], case["top"], case["E"]
    logits = torch.randn((T, E), device="cuda", generator=gen) + 0.5 * torch.randn((E,), device="cuda", generator=gen)
    best, ids = logits.topk(top, dim=1)
    ids = torch.where(torch.rand((T, top), device="cuda", generator=gen) < case["drop"], torch.full_like(ids, -1), ids)
    return ids.int().contiguous(), torch.softmax(best, dim=1).contiguous()


def prepare(case, seed):
    gen, dt, kind = _generator(seed), DTYPES[case["dtype"]], case["kind"]
    empty = lambda *shape, t=dt: torch.empty(shape, device="cuda", dtype=t)
    pitch = lambda k: (k + 127) // 128 * 128
    st = {"kind": kind}
    if kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        st["x"] = _normal(gen, (M, K + case["pad"]), dt)[:, :K]
        st["wq"], st["sw"] = _weights(gen, (), N, K)
        st["bias"] = _normal(gen, (N,), torch.float32) if case["bias"] else None
        st["c"], st["q"], st["s"] = empty(M, N), empty(M, pitch(K), t=torch.int8), empty(M, t=torch.float32)
        return st
    T, top, E, H, F = (case[k] for k in ("T", "top", "E", "H", "F"))
    n = T * top
    st["ids"], st["w"] = _router(gen, case)
    st["E"] = E
    i32 = lambda *shape: empty(*shape, t=torch.int32)
    st["sorted"] = (i32(n), i32(T, top), i32(E + 1))
    st["space"] = empty(1 << 22, t=torch.uint8)
    if kind == "route":
        st["x"], st["dx"] = _normal(gen, (T, H), dt), _normal(gen, (T, H), dt)
        st["y"], st["dy"] = _normal(gen, (n, H), dt), _normal(gen, (n, H), dt)
        st["out"] = {"rows": empty(n, H), "tokens": empty(T, H), "d_rows": empty(n, H), "d_weights": empty(T, top, t=torch.float32), "d_tokens": empty(T, H)}
    elif kind == "up":
        st["x"] = _normal(gen, (T, H), dt)
        st["wq"], st["sw"] = _weights(gen, (E,), F, H)
        st["c"], st["q"], st["s"] = empty(n, F), empty(n, pitch(H), t=torch.int8), empty(n, t=torch.float32)
    else:
        st["x"] = _normal(gen, (n, 2 * F), dt)  # gate and linear part of the rows in the experts' order
        st["wq"], st["sw"] = _weights(gen, (E,), H, F)
        st["sorted"] = tuple(t.int() for t in _order(st["ids"], E))  # the layer's first half has them
        st["q"], st["s"] = empty(n, pitch(F), t=torch.int8), empty(n, t=torch.float32)
        st["c"], st["tokens"] = empty(n, H), empty(T, H)
    return st


# ------------------------------------------------------------------ plain forms
def _order(ids, E):
    """order, position and offsets of the slots sorted by expert, slots without one behind."""
    e = ids.reshape(-1).long()
    kept = (e >= 0) & (e < E)
    e = torch.where(kept, e, torch.full_like(e, E))
    slot = torch.arange(e.numel(), device=e.device)
    hit = torch.zeros((e.numel(), E + 1), device=e.device, dtype=torch.int32)
    hit[slot, e] = 1
    upto = hit.cumsum(0)
    count = upto[-1]
    start = count.cumsum(0) - count
    row = start[e] + upto[slot, e] - 1
    order = torch.empty_like(row)
    order[row] = slot
    return order, torch.where(kept, row, -1 - row).view(ids.shape), start


def _quantised(x):
    """Codes as 32-bit numbers and the scale of each row."""
    amax = x.abs().amax(dim=-1, keepdim=True)
    most = torch.full_like(amax, 127.0)
    q = torch.round(x * torch.where(amax > 0, most / amax, amax))
    return q, amax / most


def _over_experts(q, s, offsets, wq, sw):
    """Rows of each expert times its weights; rows behind the last expert's are zero."""
    E, N = sw.shape
    n, K = q.shape
    row = torch.arange(n, device=q.device)
    e = (row[:, None] >= offsets[None, 1:]).sum(1)
    kept = e < E
    most = max(1, int((offsets[1:] - offsets[:-1]).max()))
    at = torch.where(kept, e * most + row - offsets[e.clamp(max=E)], torch.full_like(row, E * most))
    blocks = torch.zeros((E * most + 1, K), device=q.device)
    blocks[at] = q
    c = torch.bmm(blocks[:-1].view(E, most, K), wq[:, :, :K].float().transpose(1, 2)) * sw[:, None, :]
    c = torch.cat([c.view(E * most, N), torch.zeros((1, N), device=q.device)])
    return torch.where(kept[:, None], c[at] * s, torch.zeros((), device=q.device))


def _plain(st):
    if st["kind"] == "linear":
        x, K = st["x"], st["x"].shape[1]
        q, s = _quantised(x.float())
        c = (q @ st["wq"][:, :K].float().t()) * s * st["sw"]
        return {"c": (c if st["bias"] is None else c + st["bias"]).to(x.dtype)}
    E, w, x = st["E"], st["w"], st["x"]
    if st["kind"] == "down":
        _, position, offsets = st["sorted"]
        g, u = x.float().chunk(2, dim=1)
        q, s = _quantised(g / (1 + torch.exp(-g)) * u)
        rows = _over_experts(q, s, offsets.long(), st["wq"], st["sw"])
        return {"tokens": (_picked(rows, position.long()) * w[:, :, None]).sum(1).to(x.dtype)}
    order, position, offsets = _order(st["ids"], E)
    kept = position >= 0
    token = order // w.shape[1]
    mine = torch.arange(order.numel(), device=order.device) < offsets[E]
    sort = {"order": order.int(), "position": position.int(), "offsets": offsets.int()}
    if st["kind"] == "up":
        q, s = _quantised(x.float())
        return {**sort, "rows": _over_experts(q[token], s[token], offsets, st["wq"], st["sw"]).to(x.dtype)}
    zero = torch.zeros((), device=x.device)
    rows = torch.where(mine[:, None], x.float()[token], zero)
    y, dx = _picked(st["y"].float(), position), st["dx"].float()
    d_rows = torch.where(mine[:, None], dx[token] * w.reshape(-1)[order][:, None], zero)
    return {**sort, "rows": rows.to(x.dtype), "tokens": (y * w[:, :, None]).sum(1).to(x.dtype), "d_rows": d_rows.to(x.dtype),
            "d_weights": torch.where(kept, (y * dx[:, None, :]).sum(2), zero), "d_tokens": _picked(st["dy"].float(), position).sum(1).to(x.dtype)}


def _picked(rows, position):
    """The rows of each token's slots, zero for slots without an expert."""
    got = rows[position.clamp(min=0)]
    return torch.where((position >= 0)[:, :, None], got, torch.zeros((), device=rows.device, dtype=rows.dtype))


# ------------------------------------------------------------------ a pass
def run(st):
    if not own:
        return _plain(st)
    from paper_2605_06057_amd import binding as lib

    kind, x = st["kind"], st["x"]
    if kind == "linear":
        lib.lcma_i8_quantize(x, st["q"], st["s"])
        return {"c": lib.lcma_i8_gemm_nt(st["q"], st["s"], st["wq"], st["sw"], st["c"], x.shape[1], st["bias"])}
    w = st["w"]
    if kind == "down":
        _, position, offsets = st["sorted"]
        lib.lcma_i8_quantize(x, st["q"], st["s"], gated=True)
        lib.lcma_i8_gemm_experts(st["q"], st["s"], offsets, st["wq"], st["sw"], st["c"], x.shape[1] // 2)
        return {"tokens": lib.lcma_tokens_combine(st["c"], position, w, st["tokens"])}
    order, position, offsets = lib.lcma_tokens_sort(st["ids"], st["E"], *st["sorted"], workspace=st["space"])
    sort = {"order": order, "position": position, "offsets": offsets}
    if kind == "up":
        lib.lcma_i8_quantize_dispatch(x, position, st["q"], st["s"])
        return {**sort, "rows": lib.lcma_i8_gemm_experts(st["q"], st["s"], offsets, st["wq"], st["sw"], st["c"], x.shape[1])}
    out = st["out"]
    lib.lcma_tokens_dispatch(x, position, out["rows"])
    lib.lcma_tokens_combine(st["y"], position, w, out["tokens"])
    lib.lcma_tokens_combine_grad(st["dx"], st["y"], position, w, out["d_rows"], out["d_weights"])
    lib.lcma_tokens_combine(st["dy"], position, None, out["d_tokens"])
    return {**sort, **out}


# ------------------------------------------------------------------ what it cannot do without
def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": M * K * es + N * K + 4 * N * (2 if case["bias"] else 1) + M * N * es, "flops": 2.0 * M * N * K}
    T, top, E, H, F = (case[k] for k in ("T", "top", "E", "H", "F"))
    n = T * top
    if case["kind"] == "route":
        # dispatch, combine, and the gradients of both; the sort and the weights
        return {"bytes": (4 * T + 5 * n) * H * es + 20 * n + 4 * E, "flops": 5.0 * n * H}
    hit = E * (1 - (1 - top / E) ** T)  # experts that some token goes to, were they equally popular
    kept = n * (1 - case["drop"])
    if case["kind"] == "up":
        return {"bytes": T * H * es + hit * F * (H + 4) + n * F * es + 12 * n + 4 * E, "flops": 2.0 * kept * H * F}
    return {"bytes": n * 2 * F * es + hit * H * (F + 4) + T * H * es + 8 * n + 4 * E, "flops": 2.0 * kept * H * F}


# ------------------------------------------------------------------ the definition in 64 bits
def _rounded(x):
    """rint(127 x / max |x|) of each row and max |x| / 127."""
    most = x.abs().max(dim=1, keepdim=True).values
    safe = torch.where(most == 0, torch.ones_like(most), most)
    return torch.round(x * 127 / safe), most / 127


def exact(case, seed):
    st = prepare(case, seed)
    x = st["x"].double()
    if case["kind"] == "linear":
        q, s = _rounded(x)
        c = (q * s) @ (st["wq"][:, : x.shape[1]].double() * st["sw"].double()[:, None]).t()
        return {"c": c if st["bias"] is None else c + st["bias"].double()}
    T, top, E = case["T"], case["top"], case["E"]
    ids, w = st["ids"].flatten().tolist(), st["w"].double()
    by_expert = [[] for _ in range(E)]
    for slot, e in enumerate(ids):
        if 0 <= e < E:
            by_expert[e].append(slot)
    slots = torch.tensor([i for group in by_expert for i in group], device="cuda", dtype=torch.int64)
    m = slots.numel()
    token, weight = slots // top, w.flatten()[slots][:, None]
    ends = [sum(len(g) for g in by_expert[:e]) for e in range(E + 1)]

    def product(q, s):
        K = q.shape[1]
        parts = [(q[a:b] @ st["wq"][e, :, :K].double().t()) * s[a:b] * st["sw"][e].double() for e, (a, b) in enumerate(zip(ends, ends[1:]))]
        return torch.cat(parts)

    def behind(rows):  # rows of slots without an expert
        return torch.cat([rows, torch.zeros((T * top - m, rows.shape[1]), device="cuda", dtype=torch.float64)])

    if case["kind"] == "down":
        g, u = x[:m].chunk(2, dim=1)
        rows = product(*_rounded(u * g * torch.sigmoid(g)))
        return {"tokens": torch.zeros((T, rows.shape[1]), device="cuda", dtype=torch.float64).index_add_(0, token, rows * weight)}
    none = {"order": None, "position": None, "offsets": None}
    if case["kind"] == "up":
        q, s = _rounded(x)
        return {**none, "rows": behind(product(q[token], s[token]))}
    y, dx, dy = st["y"].double()[:m], st["dx"].double(), st["dy"].double()[:m]
    d_weights = torch.zeros((T * top,), device="cuda", dtype=torch.float64)
    d_weights[slots] = (dx[token] * y).sum(1)
    return {**none, "rows": behind(x[token]), "tokens": torch.zeros_like(x).index_add_(0, token, y * weight), "d_rows": behind(dx[token] * weight),
            "d_weights": d_weights.view(T, top), "d_tokens": torch.zeros_like(x).index_add_(0, token, dy)}
