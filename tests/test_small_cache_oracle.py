"""The oracle of 8-bit pages and eviction against values that come from elsewhere: torch's 8-bit type, the format's 256
codes written out, a scalar softmax and a scalar search."""
import math

import numpy as np
import pytest
import torch

from oracle import small_cache as orc


def codes():
    """The finite magnitudes of the format from its definition."""
    out = []
    for e in range(16):
        for m in range(8):
            if e == 15 and m == 7:
                continue                                   # NaN
            out.append(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return np.array(out)


def test_e4m3_rounds_to_the_nearest_code_ties_to_even():
    c = codes()
    assert c.max() == orc.E4M3_MAX and len(c) == 127
    rng = np.random.default_rng(1)
    mid = (c[1:] + c[:-1]) / 2
    x = np.concatenate([c, mid, np.nextafter(mid, 0), np.nextafter(mid, 500), rng.uniform(0, 448, 2000), np.exp(rng.uniform(-9, 6, 2000))])
    x = x[x <= 448]
    got = orc.round_e4m3(np.concatenate([x, -x]))
    best = np.abs(x[:, None] - c).min(axis=1)
    assert np.array_equal(np.abs(got[:len(x)] - x), best) and np.array_equal(got[len(x):], -got[:len(x)])
    for a, b, m in zip(c[:-1], c[1:], mid):                # a tie goes to the code with the even last bit
        i = int(np.where(c == a)[0][0])
        assert orc.round_e4m3(m) == (a if i % 2 == 0 else b)
    bf = torch.randn(4000, generator=torch.Generator().manual_seed(3)).bfloat16() * 20
    assert np.array_equal(orc.round_e4m3(bf.double().numpy()), bf.to(torch.float8_e4m3fn).double().numpy())
    assert np.isnan(orc.round_e4m3([np.inf, -np.inf, np.nan])).all()


@pytest.mark.parametrize("top,scale", [(0.0, 1.0), (448.0, 1.0), (449.0, 2.0), (224.0, 0.5), (224.5, 1.0), (1.0, 2.0 ** -8), (1.75, 2.0 ** -8),
                                       (1.76, 2.0 ** -7), (2.0 ** -130, 2.0 ** -126), (3.0e38, 2.0 ** 120)])
def test_page_scale_is_the_least_power_of_two_that_fits(top, scale):
    assert orc.page_scale([[-top, 0.0], [np.nan, np.inf]]) == scale


def test_weights_are_the_probabilities_of_a_scalar_softmax():
    rng = np.random.default_rng(5)
    d, n = 4, 5
    k, v, q = rng.standard_normal((2, 4, d)), rng.standard_normal((2, 4, d)), rng.standard_normal((1, 2, d))
    o, got = orc.attend_decode(q, [0], None, k, v, np.array([[1]]), [2], np.array([[0]]), [3], 1e4, 4)
    keys = [k[1, 0], k[1, 1], k[0, 0], k[0, 1], k[0, 2]]
    vals = [v[1, 0], v[1, 1], v[0, 0], v[0, 1], v[0, 2]]
    for h in range(2):
        e = [math.exp(sum(a * b for a, b in zip(q[0, h], key)) / math.sqrt(d)) for key in keys]
        for i in range(d):
            assert abs(o[0, h, i] - sum(x * val[i] for x, val in zip(e, vals)) / sum(e)) < 1e-12
    assert len(got[0]) == n and abs(got[0].sum() - 2) < 1e-12


def test_keep_rows():
    assert orc.keep_rows([3.0, 1.0, 2.0], 3, 0) == [0, 1, 2]
    assert orc.keep_rows([3.0, 1.0, 2.0, 9.0], 2, 1) == [0, 3]
    assert orc.keep_rows([1.0, 1.0, 1.0, 1.0], 2, 0) == [0, 1]
    assert orc.keep_rows([math.nan, 0.0, -math.inf, 5.0], 3, 0) == [1, 2, 3]
    assert orc.keep_rows([math.nan, math.nan, 4.0], 2, 0) == [0, 2]
    assert orc.keep_rows([5.0, 4.0, 3.0, 2.0], 2, 2) == [2, 3]
