"""Attention over the 4-bit cache at the ends of the ranges that it is stated for: cached values up to 2^80, scores up to 2^24."""
import numpy as np
import pytest

import kv_cases
import test_gpu_kv as kv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,new,R,D,G", [([3000, 40], [1, 1], 4, 128, 128), ([3000, 40], [2, 1], 4, 128, 32), ([1500, 37], [1, 1], 3, 256, 64),
                                            ([3000, 90], [100, 90], 1, 128, 64), ([2000, 70], [90, 70], 1, 256, 128), ([300, 20], [70, 20], 2, 64, 32)])
@pytest.mark.parametrize("spread,q_scale", [(2.0 ** 75, 2.0 ** -75), (2.0 ** -60, 2.0 ** 60), (2.0 ** 9, 2.0 ** 9)])
def test_ends_of_the_ranges(lens, new, R, D, G, spread, q_scale):
    """(2^75 a standard deviation, times 4 in every 17th feature: up to 2^80; 2^18 q k sums to 2^18 * D^0.5 * about 4 and more.  There
    fp32 scores are off by several units, which the bound allows: what is held is that outputs stay among the values.)"""
    c = kv.Cache(lens, new, 1, D, G, 16, seed=sum(lens) + D).fill(spread)
    top = max(np.abs(v).max() for v in c.v)
    assert spread > 1 or top < 2.0 ** -55
    assert spread < 2.0 ** 70 or 2.0 ** 78 < top <= 2.0 ** 80
    got = kv_cases.attend(c, R, single=max(new) == 1, q_scale=q_scale)
    assert np.isfinite(got).all() and np.abs(got).max() <= top * (1 + 2.0 ** -7)
