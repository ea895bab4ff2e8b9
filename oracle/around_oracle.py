"""CPU oracle of the operators around the layer in fp64 (plain numpy, no code
shared with the HIP path): residual norm, token sampling, accepted path."""
from __future__ import annotations

import numpy as np


def residual_norm(hidden, y, weight, eps):
    """(s, n) in fp64: s = hidden + y, n = s / sqrt(mean s^2 + eps) * weight."""
    s = np.asarray(hidden, np.float64)
    if y is not None:
        s = s + np.asarray(y, np.float64)
    size = np.sqrt((s * s).sum(axis=1, keepdims=True) / s.shape[1] + eps)
    return s, s / size * np.asarray(weight, np.float64)


def e4m3_values():
    """The 256 values of the 8-bit type (4 exponent bits of bias 7, 3 mantissa bits; 0x7f NaN)."""
    out = np.zeros(256)
    for c in range(256):
        ex, man = (c >> 3) & 15, c & 7
        v = (man / 8) * 2.0 ** -6 if ex == 0 else (1 + man / 8) * 2.0 ** (ex - 7)
        out[c] = np.nan if (c & 127) == 127 else (-v if c & 128 else v)
    return out


def sample_row(z, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """(token, prob, margin) of one row.  margin: the distance, relative to the sum of
    weights, from u and top_p's sum to the nearest border between two tokens, over what
    64-bit arithmetic may move a border by: sums of 1024 terms in a chain and exponentials
    (1e-12), n weights held to 2^-44 or, below e^-31, left out (1e-13 each of the
    largest), z / temperature rounded to 64 bits (from 2^20 on the difference to the
    largest is taken first).  Above 1 the token is certain."""
    z = np.asarray(z, np.float64)
    live = np.flatnonzero(z > -np.inf)  # drops NaN too
    if live.size == 0:
        return -1, 0.0, np.inf
    order = live[np.argsort(-z[live], kind="stable")]
    if temperature is not None and not temperature > 0:
        return int(order[0]), 1.0, np.inf
    tau = 1.0 if temperature is None else float(temperature)
    top = z[order[0]]
    with np.errstate(invalid="ignore"):
        w = np.where(z[order] == top, 1.0, np.exp((z[order] - top) / tau))
    if top_k is not None and top_k > 0:
        order, w = order[:top_k], w[:top_k]
    c = np.cumsum(w)
    margin, moved = np.inf, 1e-12 + len(w) * 1e-13 / c[-1] + (abs(top) / tau * 2.0 ** -52 if abs(top) / tau < 2 ** 20 else 0.0)
    if top_p is not None and top_p < 1:
        want = max(float(top_p), 0.0) * c[-1]
        n = 1
        while n < len(c) and c[n - 1] < want:
            n += 1
        if want > 0:
            margin = float(np.abs(c - want).min() / c[-1])
        order, w, c = order[:n], w[:n], c[:n]
    if min_p is not None and min_p > 0:
        n = max(1, int((w >= min(float(min_p), 1.0)).sum()))
        order, w, c = order[:n], w[:n], c[:n]
    u = min(max(float(u), 0.0), 1.0)
    over = np.flatnonzero(c > u * c[-1])
    j = int(over[0]) if over.size else int(np.flatnonzero(w > 0)[-1])
    if u > 0:
        margin = min(margin, float(np.abs(c[:-1] - u * c[-1]).min(initial=np.inf) / c[-1]))
    return int(order[j]), float(w[j] / c[-1]), margin / moved


def accept(token, parent, target, offsets):
    """(on_path, paths, length, bonus): walks down from each root."""
    on = np.zeros(len(token), np.uint8)
    paths, length, bonus = [], [], []
    for a, b in zip(offsets, offsets[1:]):
        walk = [a] if b > a else []
        while walk:
            kids = [t for t in range(walk[-1] + 1, b) if parent[t] == walk[-1] and token[t] == target[walk[-1]]]
            if not kids:
                break
            walk.append(kids[0])
        on[walk] = 1
        paths.append(walk)
        length.append(len(walk))
        bonus.append(int(target[walk[-1]]) if walk else -1)
    return on, paths, length, bonus


E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0])


def dequantize_q4(codes, scales):
    """[..., K / 2] codes (lower nibble first) and [..., K / 32] scales -> [..., K] fp64."""
    codes, scales = np.asarray(codes), np.asarray(scales)
    v = E2M1[np.stack([codes & 15, codes >> 4], axis=-1)].reshape(*codes.shape[:-1], -1)
    return v * np.repeat(2.0 ** (scales.astype(np.float64) - 127), 32, axis=-1)


def quantize_q4(w):
    """Codes and scales of [..., K]: the smallest scale with max|w| <= 6 of it, nearest code, ties to even."""
    w = np.asarray(w, np.float64)
    parts = w.reshape(*w.shape[:-1], -1, 32)
    largest = np.abs(parts).max(axis=-1)
    scales = np.full(largest.shape, 2, np.int64)
    for s in range(251, 1, -1):
        scales[largest > 6 * 2.0 ** (s - 127)] = np.maximum(scales[largest > 6 * 2.0 ** (s - 127)], s + 1)
    a = np.abs(parts) / 2.0 ** (scales[..., None] - 127.0)
    dist = np.abs(a[..., None] - E2M1[:8])
    nearest = dist.min(axis=-1, keepdims=True) == dist
    # of two equally near neighbours the even code
    code = np.where(nearest.sum(axis=-1) == 2, np.argmax(nearest & (np.arange(8) % 2 == 0), axis=-1),
                    np.argmax(nearest, axis=-1))
    code = (code + 8 * np.signbit(parts)).reshape(w.shape).astype(np.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), scales.astype(np.uint8)


def moe_forward(x, gate, up, down, idx, g):
    """Grouped SwiGLU FFN in fp64; gate, up [E, I, H], down [E, H, I]; routing entries outside
    [0, E) are skipped and a repeated expert counts at its first slot."""
    x = np.asarray(x, np.float64)
    out = np.zeros_like(x)
    for t, row in enumerate(idx):
        seen = set()
        for j, e in enumerate(row):
            if not 0 <= e < len(gate) or e in seen:
                continue
            seen.add(e)
            z = gate[e] @ x[t]
            with np.errstate(over="ignore"):
                out[t] += g[t][j] * (down[e] @ (z / (1 + np.exp(-z)) * (up[e] @ x[t])))
    return out
