"""The oracle of the operators around the layer against hand-worked values and
independent routines (CPU)."""
import math

import numpy as np
import pytest
import torch

from oracle import around_oracle as A


def test_norm_by_hand():
    s, n = A.residual_norm([[1.0, 2.0]], [[2.0, 2.0]], [1.0, 0.5], 0.0)
    assert np.array_equal(s, [[3.0, 4.0]])
    assert np.allclose(n, [[3 / math.sqrt(12.5), 2 / math.sqrt(12.5)]], rtol=1e-15)


def test_e4m3_values_equal_the_type():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(A.e4m3_values(), want, equal_nan=True)


@pytest.mark.parametrize("u,token", [(0.0, 2), (0.49, 2), (0.51, 0), (0.76, 3)])
def test_sample_by_hand(u, token):
    z = np.log([2.0, 1.0, 4.0, 2.0])  # sums 4, 6, 8, 9 of 9
    z[1] = -np.inf                    # then 4, 6, 8 of 8
    got, prob, _ = A.sample_row(z, u)
    assert got == token and prob == pytest.approx({2: 0.5, 0: 0.25, 3: 0.25}[token])


def test_sample_filters_by_hand():
    z = np.log([8.0, 4.0, 2.0, 1.0, 1.0])
    last = 0.999999
    assert A.sample_row(z, last)[0] == 4
    assert A.sample_row(z, last, top_k=4)[0] == 3
    assert A.sample_row(z, last, top_p=0.76)[0] == 2   # 12 of 16 do not reach it
    assert A.sample_row(z, last, top_p=0.74)[0] == 1
    assert A.sample_row(z, last, min_p=0.2)[0] == 2
    assert A.sample_row(z, last, min_p=2.0)[0] == 0
    assert A.sample_row(z, last, top_p=0.0)[0] == 0
    assert A.sample_row(z, last, temperature=0.0) == (0, 1.0, np.inf)
    assert A.sample_row(z, last, top_k=3, top_p=0.9)[0] == 2  # of 14: 12 do not reach 12.6
    assert A.sample_row([-np.inf, np.nan], 0.3)[:2] == (-1, 0.0)
    assert A.sample_row([1.0, np.inf, 5.0, np.inf], 0.7)[0] == 3


def test_accept_by_hand():
    #        0 (root)
    #   1:7   2:7   3:9       target of 0 is 7: 1, not 2
    #   4:5 under 2; 5:5, 6:6 under 1, target of 1 is 6
    token = [0, 7, 7, 9, 5, 5, 6]
    parent = [-1, 0, 0, 0, 2, 1, 1]
    target = [7, 6, 5, 1, 1, 1, 42]
    on, paths, length, bonus = A.accept(token, parent, target, [0, 7, 7])
    assert paths == [[0, 1, 6], []] and length == [3, 0] and bonus == [42, -1]
    assert on.tolist() == [1, 1, 0, 0, 0, 0, 1]


def test_q4_by_hand():
    w = np.zeros(64)
    w[:4] = 6.0, -0.25, 0.75, 5.0         # scale 1: 6, 0 (tie to even), 1, 4 (tie to even)
    w[32:35] = 6.5, 1.0, -3.0             # above 6: scale 2
    codes, scales = A.quantize_q4(w)
    assert scales.tolist() == [127, 128]
    v = A.dequantize_q4(codes, scales)
    assert v[:4].tolist() == [6.0, 0.0, 1.0, 4.0] and np.signbit(v[1])
    assert v[32:35].tolist() == [6.0, 1.0, -3.0]
    assert codes[0] == 7 | (8 << 4) and codes[1] == 2 | (6 << 4)


def test_q4_nearest():
    rng = np.random.default_rng(0)
    w = rng.standard_normal((50, 96)) * 2.0 ** rng.integers(-20, 20, (50, 1))
    v = A.dequantize_q4(*A.quantize_q4(w))
    scale = np.repeat(2.0 ** np.ceil(np.log2(np.abs(w).reshape(50, -1, 32).max(-1) / 6)), 32, axis=-1)
    best = np.abs(w[..., None] - scale[..., None] * A.E2M1).min(-1)
    assert np.array_equal(np.abs(w - v), best)


def test_forward_equals_dense_formula():
    rng = np.random.default_rng(1)
    x, g, u, d = (rng.standard_normal(s) for s in ((3, 8), (4, 6, 8), (4, 6, 8), (4, 8, 6)))
    idx, gate = [[0, 2], [3, 3], [-1, 9]], np.float64([[0.5, 0.25], [1.0, 7.0], [1.0, 1.0]])
    ffn = lambda e, v: d[e] @ ((g[e] @ v) / (1 + np.exp(-(g[e] @ v))) * (u[e] @ v))  # noqa: E731
    want = np.stack([0.5 * ffn(0, x[0]) + 0.25 * ffn(2, x[0]), ffn(3, x[1]), np.zeros(8)])
    assert np.allclose(A.moe_forward(x, g, u, d, idx, gate), want, rtol=1e-13)
