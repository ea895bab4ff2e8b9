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
