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
    """(token, prob, margin) of one row; margin: the distance, relative to the sum of
    weights, from u and top_p's sum to the nearest border between two tokens."""
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
    margin = np.inf
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
    return int(order[j]), float(w[j] / c[-1]), margin


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
