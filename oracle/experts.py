"""Plain 64-bit (whole numbers: exact) forms of the 8-bit-integer linear layer and of the tokens' way to their experts and back, in numpy,
sharing no code with the library.  Matrices are float64 arrays that hold the stored values."""
from __future__ import annotations

import numpy as np


def i8_quantize(x: np.ndarray):
    """Codes (int8) and scales (float32) of the rows of x (float64 holding fp32 / fp16 / bf16 values): the arithmetic is defined in fp32, so the
    codes are too.  A row of zeros has scale and codes 0, one with an infinity or a NaN codes 0 and amax / 127 for its scale."""
    x = x.astype(np.float32)
    q = np.zeros(x.shape, np.int8)
    s = np.zeros(x.shape[0], np.float32)
    for r, row in enumerate(x):
        if row.size == 0:
            continue
        amax = np.float32(np.nan) if np.isnan(row).any() else np.abs(row).max()
        s[r] = amax / np.float32(127)
        if amax > 0 and np.isfinite(amax):
            up = np.float32(2.0) ** 100 if amax < np.float32(2.0) ** -100 else np.float32(1)
            inv = np.float32(127) / (amax * up)
            q[r] = np.rint((row * up) * inv).astype(np.int8)
    return q, s


def silu_gate(x: np.ndarray) -> np.ndarray:
    """silu(first half) * second half of every row, in 64 bits."""
    g, u = np.split(x.astype(np.float64), 2, axis=1)
    return g / (1 + np.exp(-g)) * u


def i8_gemm(aq, sa, wq, sw, bias=None):
    """sa[m] sw[n] sum_k aq[m][k] wq[n][k] + bias[n]: the sum in whole numbers, the rest in 64 bits."""
    c = (aq.astype(np.float64) @ wq.astype(np.float64).T) * sa.astype(np.float64)[:, None] * sw.astype(np.float64)  # (sums below 2^53: exact)
    return c if bias is None else c + bias.astype(np.float64)


def i8_gemm_experts(aq, sa, offsets, wq, sw, bias=None):
    c = np.zeros((aq.shape[0], wq.shape[1]))
    for e in range(wq.shape[0]):
        a, b = offsets[e], offsets[e + 1]
        c[a:b] = i8_gemm(aq[a:b], sa[a:b], wq[e], sw[e], None if bias is None else bias[e])
    return c


def tokens_sort(ids: np.ndarray, experts: int):
    """order, position, offsets of the slots of ids (tokens x top_k)."""
    flat = ids.reshape(-1)
    groups = [[] for _ in range(experts + 1)]
    for slot, e in enumerate(flat.tolist()):
        groups[e if 0 <= e < experts else experts].append(slot)
    order = np.array([s for g in groups for s in g], np.int32)
    position = np.zeros(flat.size, np.int32)
    position[order] = np.arange(flat.size, dtype=np.int32)
    offsets = np.cumsum([0] + [len(g) for g in groups[:experts]]).astype(np.int32)
    position = np.where(position < offsets[experts], position, -1 - position)
    return order, position.reshape(ids.shape), offsets


def tokens_dispatch(x, position):
    y = np.zeros((position.size, x.shape[1]))
    for (t, j), row in np.ndenumerate(position):
        if row >= 0:
            y[row] = x[t]
    return y


def tokens_combine(y, position, weights=None):
    x = np.zeros((position.shape[0], y.shape[1]))
    for (t, j), row in np.ndenumerate(position):
        if row >= 0:
            x[t] += (1.0 if weights is None else float(weights[t, j])) * y[row]
    return x


def tokens_combine_grad(dx, y, position, weights):
    dy, dw = np.zeros((position.size, dx.shape[1])), np.zeros(position.shape)
    for (t, j), row in np.ndenumerate(position):
        if row >= 0:
            dy[row] = float(weights[t, j]) * dx[t]
            dw[t, j] = dx[t] @ y[row]
    return dy, dw
