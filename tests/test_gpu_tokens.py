"""Tokens sorted by expert and back, and the gradients of both, against the plain forms of oracle/experts.py."""
import numpy as np
import pytest

import lcma_inputs as inp
from oracle import experts as X

pytestmark = pytest.mark.gpu

HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def _store(rng, shape, dt):
    import gpu_util as G
    stored = inp.store(rng.standard_normal(shape), dt)
    return G.to_device(stored, dt), inp.widen(stored, dt).astype(np.float64)


def _host(t, dt):
    import gpu_util as G
    return G.to_host_f64(t, dt).astype(np.float64)


def _view(rows, cols, dt, pad):
    import torch
    td = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dt]
    whole = torch.full((rows + 2, cols + 2 * pad), float("nan"), dtype=td, device="cuda")
    return whole, whole[1:1 + rows, pad:pad + cols]


def _untouched(whole, rows, cols, pad):
    import torch
    outside = torch.ones(whole.shape, dtype=torch.bool, device="cuda")
    outside[1:1 + rows, pad:pad + cols] = False
    return torch.isnan(whole[outside]).all().item()


# ------------------------------------------------------------------ sort
def _sort_case(ids, E):
    import torch
    from paper_2605_06057_amd import binding as B
    tokens, top_k = ids.shape
    n = ids.size
    need = B.lcma_tokens_sort_workspace_bytes(tokens, top_k, E)
    guard = lambda size: torch.full((size + 2,), 123456789, dtype=torch.int32, device="cuda")
    order, position, offsets, space = guard(n), guard(n), guard(E + 1), guard(need // 4)
    B.lcma_tokens_sort(torch.from_numpy(ids).cuda(), E, order[1:1 + n], position[1:1 + n].view(tokens, top_k), offsets[1:2 + E], space[1:1 + need // 4])
    torch.cuda.synchronize()
    for t in (order, position, offsets, space):
        assert t[0].item() == 123456789 and t[-1].item() == 123456789, "wrote outside its output"
    want = X.tokens_sort(ids, E)
    assert np.array_equal(offsets[1:2 + E].cpu().numpy(), want[2])
    assert np.array_equal(order[1:1 + n].cpu().numpy(), want[0]) and np.array_equal(position[1:1 + n].cpu().numpy().reshape(ids.shape), want[1])


@pytest.mark.parametrize("E", [1, 2, 7, 8, 60, 64, 65, 255, 256, 1000, 1024])
@pytest.mark.parametrize("tokens,top_k", [(1, 1), (1, 8), (5, 3), (64, 1), (65, 1), (513, 1), (1000, 4), (1365, 3), (4096, 1), (4097, 1), (9001, 2), (70000, 1)])
def test_sort(tokens, top_k, E):
    rng = np.random.default_rng(tokens * top_k + E)
    _sort_case(rng.integers(0, E, (tokens, top_k)).astype(np.int32), E)


@pytest.mark.parametrize("tokens", [3, 700, 5000])
@pytest.mark.parametrize("what", ["some without", "all without", "one expert", "last expert", "alternating", "descending", "far out"])
def test_sort_of_unusual_numbers(tokens, what):
    rng = np.random.default_rng(tokens)
    E, top_k = 9, 2
    ids = rng.integers(0, E, (tokens, top_k))
    slots = np.arange(tokens * top_k).reshape(tokens, top_k)
    ids = {"some without": np.where(rng.random(ids.shape) < 0.3, -1, ids), "all without": np.full_like(ids, -1), "one expert": np.zeros_like(ids),
           "last expert": np.full_like(ids, E - 1), "alternating": slots % E, "descending": (tokens * top_k - 1 - slots) * E // (tokens * top_k),
           "far out": rng.choice([-2 ** 31, 2 ** 31 - 1, E, -1, 3, 1 << 20], ids.shape)}[what]
    _sort_case(ids.astype(np.int32), E)


def test_sort_of_no_tokens():
    import torch
    from paper_2605_06057_amd import binding as B
    order, position, offsets = B.lcma_tokens_sort(torch.empty((0, 2), dtype=torch.int32, device="cuda"), 5)
    assert order.numel() == 0 and position.shape == (0, 2) and offsets.tolist() == [0] * 6


def test_sort_of_many_slots():
    """More blocks than a wave has lanes; the plain order by torch's stable sort."""
    import torch
    from paper_2605_06057_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(3)
    ids = torch.randint(0, 40, (300001, 1), device="cuda", generator=gen).int()
    order, position, offsets = B.lcma_tokens_sort(ids, 40)
    want = torch.sort(ids.flatten(), stable=True)[1]
    assert torch.equal(order.long(), want) and torch.equal(order[position.flatten().long()].long(), torch.arange(300001, device="cuda"))
    assert torch.equal(offsets.long(), torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), torch.bincount(ids.flatten(), minlength=40).cumsum(0)]))


# ------------------------------------------------------------------ rows
ROWS = [(1, 1, 1, 0), (1, 2, 3, 0), (3, 2, 4, 0), (5, 3, 7, 1), (4, 1, 8, 0), (9, 2, 9, 0), (17, 8, 64, 0), (33, 2, 129, 3), (6, 6, 520, 8), (40, 4, 1543, 0), (5, 5, 2048, 0),
        (3, 2, 4100, 1), (2, 8, 9001, 0), (300, 9, 40, 0)]


def _routing(rng, tokens, top_k, share):
    import torch
    from paper_2605_06057_amd import binding as B
    ids = np.where(rng.random((tokens, top_k)) < share, -1, rng.integers(0, 6, (tokens, top_k))).astype(np.int32)
    _, position, offsets = B.lcma_tokens_sort(torch.from_numpy(ids).cuda(), 6)
    w = rng.uniform(-1, 1, (tokens, top_k)).astype(np.float32)
    return position, position.cpu().numpy(), int(offsets[-1]), w, torch.from_numpy(w).cuda()


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("share", [0.0, 0.3, 1.0])
@pytest.mark.parametrize("tokens,top_k,H,pad", ROWS)
def test_rows(dt, share, tokens, top_k, H, pad):
    import torch
    from paper_2605_06057_amd import binding as B
    rng = np.random.default_rng(tokens * 1000 + H)
    position, pos, kept, w, weights = _routing(rng, tokens, top_k, share)
    n = tokens * top_k
    # dispatch: a copy, bit for bit
    x, x64 = _store(rng, (tokens, H), dt)
    whole_x, xv = _view(tokens, H, dt, pad)
    xv.copy_(x)
    whole, y = _view(n, H, dt, pad)
    B.lcma_tokens_dispatch(xv, position, y)
    assert np.array_equal(_host(y, dt), X.tokens_dispatch(x64, pos)) and _untouched(whole, n, H, pad)
    # combine, with weights and without: fp32 products and sums (2^-24 of a magnitude each, top_k of both), one rounding
    rows, rows64 = _store(rng, (n, H), dt)
    whole_r, rv = _view(n, H, dt, pad)
    rv.copy_(rows)
    rv[kept:] = float("nan")  # never read
    rows64[kept:] = 0
    for wt, wh in ((weights, w), (None, None)):
        whole, out = _view(tokens, H, dt, pad)
        B.lcma_tokens_combine(rv, position, wt, out)
        want = X.tokens_combine(rows64, pos, wh)
        size = X.tokens_combine(np.abs(rows64), pos, None if wh is None else np.abs(wh))
        room = size * (top_k + 1) * 2.0 ** -24 + np.abs(want) * 1.001 * HALF_ULP[dt] + 2.0 ** -25
        assert np.all(np.abs(_host(out, dt) - want) <= room) and _untouched(whole, tokens, H, pad)
    # the gradient of combine: a rounded product, and a dot product of H terms in fp32
    whole, dy = _view(n, H, dt, pad)
    dw = torch.full((tokens, top_k), float("nan"), device="cuda")
    B.lcma_tokens_combine_grad(xv, rv, position, weights, dy, dw)
    want_y, want_w = X.tokens_combine_grad(x64, rows64, pos, w)
    assert np.all(np.abs(_host(dy, dt) - want_y) <= np.abs(want_y) * (2.0 ** -24 + 1.001 * HALF_ULP[dt]) + 2.0 ** -25) and _untouched(whole, n, H, pad)
    _, size = X.tokens_combine_grad(np.abs(x64), np.abs(rows64), pos, w)
    assert np.all(np.abs(dw.cpu().numpy() - want_w) <= size * (H + 1) * 2.0 ** -24)


@pytest.mark.parametrize("tokens,top_k,H", [(7, 2, 33), (20, 3, 256)])
def test_gradients_against_differences(tokens, top_k, H):
    """<dX, combine(Y, w)> is linear in Y and in w, so a difference over any step is the gradient times it, up to rounding: fp32 values of
    magnitude about 1, sums of at most tokens * H terms, bound 2^-20 of the sum of the magnitudes.  So is <dY, dispatch(X)> in X."""
    import torch
    from paper_2605_06057_amd import binding as B
    rng = np.random.default_rng(H)
    position, _, kept, _, w = _routing(rng, tokens, top_k, 0.2)
    n = tokens * top_k
    make = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda()
    y, dx, dir_y, dir_w = make(n, H), make(tokens, H), make(n, H), make(tokens, top_k)
    dy, dw = B.lcma_tokens_combine_grad(dx, y, position, w)
    loss = lambda a, b: (B.lcma_tokens_combine(a, position, b).double() * dx.double()).sum().item()
    size = (B.lcma_tokens_combine(y.abs() + dir_y.abs(), position, w.abs() + dir_w.abs()).double() * dx.double().abs()).sum().item()
    assert abs(loss(y + dir_y, w) - loss(y - dir_y, w) - 2 * (dy.double() * dir_y.double()).sum().item()) <= size * 2.0 ** -20
    assert abs(loss(y, w + dir_w) - loss(y, w - dir_w) - 2 * (dw.double() * dir_w.double()).sum().item()) <= size * 2.0 ** -20
    x, dir_x, g = make(tokens, H), make(tokens, H), make(n, H)
    dxg = B.lcma_tokens_combine(g, position)
    moved = lambda a: (B.lcma_tokens_dispatch(a, position).double() * g.double()).sum().item()
    size = (B.lcma_tokens_dispatch(x.abs() + dir_x.abs(), position).double() * g.double().abs()).sum().item()
    assert abs(moved(x + dir_x) - moved(x - dir_x) - 2 * (dxg.double() * dir_x.double()).sum().item()) <= size * 2.0 ** -20


def test_on_a_stream_of_its_own_and_in_a_graph():
    """The whole layer on another stream than the default one, then captured: every replay gives what the eager calls give on the inputs of then."""
    import torch
    from paper_2605_06057_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(11)
    T, top_k, E, H, F = 37, 2, 5, 256, 384
    pitch = B.lcma_i8_code_pitch
    w1, s1 = torch.randint(-127, 128, (E, 2 * F, pitch(H)), device="cuda", generator=gen).to(torch.int8), torch.rand((E, 2 * F), device="cuda", generator=gen) / 500
    w2, s2 = torch.randint(-127, 128, (E, H, pitch(F)), device="cuda", generator=gen).to(torch.int8), torch.rand((E, H), device="cuda", generator=gen) / 500
    x, ids = torch.randn((T, H), device="cuda", generator=gen).bfloat16(), torch.randint(-1, E, (T, top_k), device="cuda", generator=gen).int()
    w = torch.rand((T, top_k), device="cuda", generator=gen)
    n = T * top_k
    new = lambda *shape, t=torch.bfloat16: torch.empty(shape, device="cuda", dtype=t)
    buffers = dict(order=new(n, t=torch.int32), position=new(T, top_k, t=torch.int32), offsets=new(E + 1, t=torch.int32), q1=new(n, pitch(H), t=torch.int8),
                   s1=new(n, t=torch.float32), h=new(n, 2 * F), q2=new(n, pitch(F), t=torch.int8), s2=new(n, t=torch.float32), y=new(n, H), out=new(T, H))

    def layer(b):
        B.lcma_tokens_sort(ids, E, b["order"], b["position"], b["offsets"])
        B.lcma_i8_quantize_dispatch(x, b["position"], b["q1"], b["s1"])
        B.lcma_i8_gemm_experts(b["q1"], b["s1"], b["offsets"], w1, s1, b["h"], H)
        B.lcma_i8_quantize(b["h"], b["q2"], b["s2"], gated=True)
        B.lcma_i8_gemm_experts(b["q2"], b["s2"], b["offsets"], w2, s2, b["y"], F)
        return B.lcma_tokens_combine(b["y"], b["position"], w, b["out"])

    want = layer(buffers).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x.add_(0)  # work of this stream in front
        buffers["out"].fill_(float("nan"))
        got = layer(buffers)
    side.synchronize()
    assert torch.equal(got, want) and torch.isfinite(want).all().item()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(buffers)
    other = {k: torch.empty_like(v) for k, v in buffers.items()}
    for k in range(4):
        x.copy_(torch.randn((T, H), device="cuda", generator=gen))
        ids.copy_(torch.randint(-1, E, (T, top_k), device="cuda", generator=gen))
        want = layer(other).clone()
        torch.cuda.synchronize()
        buffers["out"].fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(buffers["out"], want), f"replay {k}"


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_many_tokens(dt):
    """More tokens than a grid has in its second dimension; the plain forms by torch's indexing."""
    import torch
    from paper_2605_06057_amd import binding as B
    td = {"f32": torch.float32, "bf16": torch.bfloat16}[dt]
    gen = torch.Generator(device="cuda").manual_seed(6)
    T, top_k, H = 70001, 3, 24
    ids = torch.randint(-1, 40, (T, top_k), device="cuda", generator=gen).int()
    x, w = torch.randn((T, H), device="cuda", generator=gen).to(td), torch.rand((T, top_k), device="cuda", generator=gen)
    order, position, offsets = B.lcma_tokens_sort(ids, 40)
    kept = int(offsets[-1])
    rows = B.lcma_tokens_dispatch(x, position)
    assert torch.equal(rows[:kept], x[order[:kept].long() // top_k]) and (rows[kept:] == 0).all().item()
    picked = torch.where((position >= 0)[:, :, None], rows.double()[position.clamp(min=0).long()], 0.0)
    got, want = B.lcma_tokens_combine(rows, position, w).double(), (picked * w.double()[:, :, None]).sum(1)
    assert ((got - want).abs() <= picked.abs().sum(1) * 4 * 2.0 ** -24 + want.abs() * 1.001 * HALF_ULP[dt] + 2.0 ** -25).all().item()
    dy, dw = B.lcma_tokens_combine_grad(x, rows, position, w)
    assert ((dw.double() - (picked * x.double()[:, None]).sum(2)).abs() <= (picked * x.double()[:, None]).abs().sum(2) * (H + 1) * 2.0 ** -24).all().item()
    want = (x.double()[:, None] * w.double()[:, :, None])[position >= 0]
    assert ((dy.double()[position[position >= 0].long()] - want).abs() <= want.abs() * (2.0 ** -24 + 1.001 * HALF_ULP[dt]) + 2.0 ** -25).all().item() and (dy[kept:] == 0).all().item()


def test_no_tokens_and_no_columns():
    import torch
    from paper_2605_06057_amd import binding as B
    none = torch.empty((0, 2), dtype=torch.int32, device="cuda")
    x, w = torch.empty((0, 16), device="cuda"), torch.empty((0, 2), device="cuda")
    assert B.lcma_tokens_dispatch(x, none).shape == (0, 16) and B.lcma_tokens_combine(x, none, w).shape == (0, 16)
    assert [t.shape for t in B.lcma_tokens_combine_grad(x, x, none, w)] == [(0, 16), (0, 2)]
    assert [t.shape for t in B.lcma_i8_quantize_dispatch(x, none)] == [(0, 128), (0,)]
    _, position, _ = B.lcma_tokens_sort(torch.zeros((3, 2), dtype=torch.int32, device="cuda"), 2)
    empty, w = torch.empty((3, 0), device="cuda"), torch.ones((3, 2), device="cuda")
    assert B.lcma_tokens_dispatch(empty, position).shape == (6, 0)
    _, dw = B.lcma_tokens_combine_grad(empty, torch.empty((6, 0), device="cuda"), position, w)
    assert (dw == 0).all().item()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,top_k,H", [(5, 3, 2), (6, 5, 40), (4, 2, 4100)])
def test_positions_that_name_no_row(dt, tokens, top_k, H):
    """The row behind the last one, as a slot's own and as that of a slot without an expert: neither read nor written."""
    import torch
    from paper_2605_06057_amd import binding as B
    rng = np.random.default_rng(H)
    n = tokens * top_k
    pos = rng.permutation(n).astype(np.int32).reshape(tokens, top_k)
    gone = pos[[0, -1], [top_k - 1, 0]]  # (the rows that no slot has any more)
    pos[0, top_k - 1], pos[-1, 0] = n, -1 - n
    none = np.where((pos < 0) | (pos >= n), -1, pos)
    position = torch.from_numpy(pos).cuda()
    x, x64 = _store(rng, (tokens, H), dt)
    w = rng.uniform(-1, 1, (tokens, top_k)).astype(np.float32)
    weights, named = torch.from_numpy(w).cuda(), np.setdiff1d(np.arange(n), gone)
    rows, rows64 = _store(rng, (n, H), dt)
    whole_r, rv = _view(n, H, dt, 0)
    rv.copy_(rows)
    whole, y = _view(n, H, dt, 0)
    B.lcma_tokens_dispatch(x, position, y)
    want = np.full((n, H), np.nan)
    want[none[none >= 0]] = x64[np.nonzero(none >= 0)[0]]
    assert np.array_equal(_host(y, dt), want, equal_nan=True) and _untouched(whole, n, H, 0)
    out = B.lcma_tokens_combine(rv, position, weights)
    wz = np.where(none < 0, 0, w).astype(np.float64)
    taken = rows64[np.maximum(none, 0)]
    want, size = (wz[..., None] * taken).sum(1), np.abs(wz[..., None] * taken).sum(1)
    assert np.all(np.abs(_host(out, dt) - want) <= size * (top_k + 1) * 2.0 ** -24 + np.abs(want) * 1.001 * HALF_ULP[dt] + 2.0 ** -25)
    whole, dy = _view(n, H, dt, 0)
    _, dw = B.lcma_tokens_combine_grad(x, rv, position, weights, dy)
    got, product = _host(dy, dt), w[..., None].astype(np.float64) * x64[:, None]
    assert np.isnan(got[gone]).all() and np.isfinite(got[named]).all() and _untouched(whole, n, H, 0)
    room = np.abs(product) * (2.0 ** -24 + 1.001 * HALF_ULP[dt]) + 2.0 ** -25
    assert np.all((np.abs(got[np.maximum(none, 0)] - product) <= room)[none >= 0])
    want, size = (taken * x64[:, None]).sum(-1), np.abs(taken * x64[:, None]).sum(-1)
    got = dw.cpu().numpy()
    assert np.all(got[none < 0] == 0) and np.all((np.abs(got - want) <= size * (H + 1) * 2.0 ** -24)[none >= 0])


# ------------------------------------------------------------------ rows that pass the caches by
def _large(dt, T, top_k, H, pad):
    """Dispatch, combine with weights and without, and the gradient of it, against torch's indexing in 64 bits; slots without an expert, NaN in the rows behind
    and around every output."""
    import torch
    from paper_2605_06057_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(T + H)
    n = T * top_k
    ids = torch.randint(-1, 7, (T, top_k), device="cuda", generator=gen).int()
    order, position, offsets = B.lcma_tokens_sort(ids, 7)
    kept = int(offsets[-1])
    w = torch.rand((T, top_k), device="cuda", generator=gen) * 2 - 1

    def filled(rows):
        whole, view = _view(rows, H, dt, pad)
        view.copy_(torch.randn((rows, H), device="cuda", generator=gen))
        return view

    x, rows = filled(T), filled(n)
    rows[kept:] = float("nan")
    token, has = order.long() // top_k, (position >= 0)[:, :, None]
    whole, y = _view(n, H, dt, pad)
    B.lcma_tokens_dispatch(x, position, y)
    assert torch.equal(y[:kept], x[token[:kept]]) and (y[kept:] == 0).all().item() and _untouched(whole, n, H, pad)
    picked = torch.where(has, rows[position.clamp(min=0).long()].double(), 0.0)
    for weights in (w, None):
        whole, out = _view(T, H, dt, pad)
        B.lcma_tokens_combine(rows, position, weights, out)
        each = picked if weights is None else picked * w.double()[:, :, None]
        want = each.sum(1)
        assert ((out.double() - want).abs() <= each.abs().sum(1) * (top_k + 1) * 2.0 ** -24 + want.abs() * 1.001 * HALF_ULP[dt] + 2.0 ** -25).all().item()
        assert _untouched(whole, T, H, pad)
        del each
    whole, dy = _view(n, H, dt, pad)
    _, dw = B.lcma_tokens_combine_grad(x, rows, position, w, dy)
    picked *= x.double()[:, None]
    assert ((dw.double() - picked.sum(2)).abs() <= picked.abs().sum(2) * (H + 1) * 2.0 ** -24).all().item()
    want = x.double()[token[:kept]] * w.double().flatten()[order[:kept].long()][:, None]
    assert ((dy[:kept].double() - want).abs() <= want.abs() * (2.0 ** -24 + 1.001 * HALF_ULP[dt]) + 2.0 ** -25).all().item()
    assert (dy[kept:] == 0).all().item() and _untouched(whole, n, H, pad)


# Written rows pass the caches by from 64 MiB on, read ones in expert order from 256 MiB on: 3 slots a token: the writes alone, 4: both, 8: the reads alone (combine).
# Rows of more than 128 vectors (odd and whole ones) and of fewer, which the gradient gives to a wave.
@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("row,pad", [(6172, 3), (6176, 0), (2036, 1), (2048, 8)])
@pytest.mark.parametrize("top_k", [3, 4, 8])
def test_rows_past_the_caches(dt, row, pad, top_k):
    es = 4 if dt == "f32" else 2
    H = (row // es) if row % 16 == 0 else row // es - (row // es + 1) % 2  # (an odd number of elements)
    mib = 65 if top_k < 8 else 33
    T = (mib << 20) // (H * es) + 1
    written, read = T * H * es >> 20, T * top_k * H * es >> 20
    assert (written >= 64, read >= 256) == {3: (True, False), 4: (True, True), 8: (False, True)}[top_k] and (H * es > 2048) == (row > 2048)
    _large(dt, T, top_k, H, pad)


# ------------------------------------------------------------------ more tokens than a launch holds along one dimension
def test_very_many_tokens():
    """2^24 tokens of short rows."""
    import torch
    from paper_2605_06057_amd import binding as B
    T, H = (1 << 24) + 5, 9
    x = (torch.arange(T * H, device="cuda", dtype=torch.int32) % 251).bfloat16().view(T, H)
    position = torch.flip(torch.arange(T, device="cuda", dtype=torch.int32), (0,)).view(T, 1)
    y = B.lcma_tokens_dispatch(x, position)
    assert torch.equal(y, x.flip(0))
    assert torch.equal(B.lcma_tokens_combine(y, position), x)
    w = torch.full((T, 1), 0.5, device="cuda")
    dy, dw = B.lcma_tokens_combine_grad(x, y, position, w)
    assert torch.equal(dy, (x * 0.5).flip(0)) and torch.equal(dw[:, 0], (x.double() ** 2).sum(1).float())


def test_very_many_long_tokens():
    """More tokens of long rows than 2^20 work-groups, which a launch spreads over two dimensions."""
    import torch
    from paper_2605_06057_amd import binding as B
    T, H = (1 << 20) + 3, 4089
    x = torch.zeros((T, H), dtype=torch.bfloat16, device="cuda")
    number = (torch.arange(T, device="cuda") % 100 + 1).bfloat16()
    x[:, 0], x[:, 2051], x[:, H - 1] = number, 2, -number
    position = torch.flip(torch.arange(T, device="cuda", dtype=torch.int32), (0,)).view(T, 1)
    y = B.lcma_tokens_dispatch(x, position)
    assert torch.equal(y, x.flip(0))
    assert torch.equal(B.lcma_tokens_combine(y, position), x)
    w = torch.full((T, 1), 0.5, device="cuda")
    dy, dw = B.lcma_tokens_combine_grad(x, y, position, w)
    assert torch.equal(dy, (y * 0.5)) and torch.equal(dw[:, 0], 2 * number.float() ** 2 + 4)
