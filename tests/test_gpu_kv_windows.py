"""Attention over the 4-bit cache with a window where a sequence's last tile of rows goes through fewer steps than an earlier one, and
sequences are cut into shares; and calls of 33 to 64 rows, or of 8 groups, at the bound of the kernel that they go to."""
import pytest

import kv_cases
import test_gpu_kv as kv

pytestmark = pytest.mark.gpu


CUT = [  # lens, new, heads, R, D, G, window, sinks
    ([8192], [5], 1, 4, 128, 128, 512, 0),
    ([2000], [16], 8, 2, 128, 128, 1000, 0),
    ([8192], [9], 2, 2, 128, 128, 4096, 0),
    ([8192] * 4, [9] * 4, 2, 2, 128, 128, 4096, 0),
    ([3000] * 4, [64] * 4, 8, 8, 128, 128, 1024, 4),
    ([2050], [385], 32, 1, 128, 128, 1024, 0),
    ([4100] * 4, [200] * 4, 8, 2, 128, 128, 512, 4),
    ([3000 - b for b in range(70)], [17] * 70, 1, 1, 64, 64, 600, 0),
    ([2500 - 7 * b for b in range(66)], [5 - b % 3 for b in range(66)], 1, 4, 128, 64, 500, 3),
    ([4000], [9], 1, 2, 256, 64, 1500, 2),
    ([4000, 3500], [300, 140], 1, 1, 256, 128, 800, 5),
]


@pytest.mark.parametrize("lens,new,heads,R,D,G,window,sinks", CUT)
def test_cut_tiles_of_unlike_spans(lens, new, heads, R, D, G, window, sinks):
    c = kv.Cache(lens, new, heads, D, G, 16, seed=sum(lens) + D).fill()
    kv_cases.attend(c, R, window=window, sinks=sinks)


@pytest.mark.parametrize("over", [0, 1, 31, 33, 63])
@pytest.mark.parametrize("new,R,window,sinks", [(17, 1, 512, 0), (5, 4, 991, 2), (130, 1, 1000, 0), (129, 2, 2033, 70)])
def test_window_on_any_token_of_a_tile(over, new, R, window, sinks):
    c = kv.Cache([4096 + over, 2048 + over], [new, new], 2, 128, 128, 32, seed=over + new).fill()
    kv_cases.attend(c, R, window=window, sinks=sinks)
    c = kv.Cache([4096 + over], [new], 1, 64, 32, 32, seed=over + new).fill()
    kv_cases.attend(c, R, window=window, sinks=sinks)


RULE = [  # lens, new, heads, R, D, G, page, window, cap
    ([33], [33], 1, 1, 128, 128, 16, 0, 0.0),
    ([700, 40], [64, 40], 3, 1, 64, 64, 16, 0, 0.0),
    ([3000, 2800], [34, 50], 1, 1, 64, 32, 64, 1500, 0.0),
    ([900, 2000, 40], [15, 16, 9], 1, 4, 256, 128, 32, 500, 0.0),
    ([900, 2000, 40], [64, 1, 40], 2, 1, 128, 128, 16, 0, 20.0),
    ([500, 60], [4, 2], 2, 16, 128, 64, 16, 0, 0.0),
    ([500, 60], [4, 2], 2, 8, 128, 32, 16, 0, 0.0),       # 32 rows of 4 groups
    ([500, 60], [33, 2], 2, 1, 128, 32, 16, 0, 0.0),      # one more
    ([500, 60], [2, 2], 2, 4, 256, 32, 16, 0, 0.0),       # 8 rows of 8 groups
    ([500, 60], [3, 3], 2, 3, 256, 32, 16, 0, 0.0),       # one more
]


@pytest.mark.parametrize("lens,new,heads,R,D,G,page,window,cap", RULE)
def test_rows_at_the_bound_of_their_kernel(lens, new, heads, R, D, G, page, window, cap):
    c = kv.Cache(lens, new, heads, D, G, page, seed=sum(lens) + D).fill()
    kv_cases.attend(c, R, window=window, cap=cap)
