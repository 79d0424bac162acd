"""Attention over the 4-bit cache with bounds on the scores from far below them to the largest that is taken."""
import pytest

import kv_cases
import test_gpu_kv as kv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cap", [2.0 ** -20, 1e-3, 1.0, 200.0, 1024.0])
@pytest.mark.parametrize("lens,new,R,D,G", [([300, 40], [1, 1], 4, 128, 128), ([300, 40], [2, 1], 4, 128, 32), ([150, 37], [1, 1], 3, 256, 64),
                                            ([300, 90], [100, 90], 1, 128, 64), ([200, 70], [90, 70], 1, 256, 128), ([300, 20], [70, 20], 2, 64, 32)])
def test_bounds_far_from_the_scores(lens, new, R, D, G, cap):
    """(a bound's 2^-22, 2^-12 at 1024, is below what the scores' own sums may be off here)"""
    for q_scale in (1.0, 30.0):
        c = kv.Cache(lens, new, 1, D, G, 16, seed=sum(lens) + D).fill()
        kv_cases.attend(c, R, single=max(new) == 1, cap=cap, q_scale=q_scale)
