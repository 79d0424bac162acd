"""Attention over the 4-bit cache of sequences that are longer than their row of the table: what lies past it is absent, also where the
table ends inside a tile of tokens."""
import pytest

import kv_cases
import test_gpu_kv as kv

pytestmark = pytest.mark.gpu


PAST = [  # table entries, page, lengths, new, heads, R, D, G, window, sinks, cap
    (3, 16, [64, 49, 200], [1, 1, 1], 2, 4, 128, 128, 0, 0, 0.0),
    (1, 16, [100, 17], [1, 1], 1, 1, 64, 32, 0, 0, 0.0),
    (5, 16, [95, 81], [6, 4], 1, 4, 128, 64, 30, 3, 0.0),         # positions on both sides of the end; a window that reaches back over it
    (3, 16, [300, 50], [3, 3], 1, 2, 256, 32, 0, 0, 20.0),
    (77, 16, [1300, 1240], [1, 1], 1, 2, 128, 32, 0, 0, 0.0),     # in shares
    (3, 16, [64, 49, 130], [40, 49, 70], 1, 2, 128, 128, 0, 0, 0.0),
    (3, 32, [97, 128, 400], [90, 70, 100], 2, 1, 128, 64, 0, 0, 0.0),
    (5, 16, [300, 81], [250, 80], 1, 1, 64, 64, 60, 5, 0.0),
    (5, 16, [300, 81], [250, 80], 1, 1, 64, 64, 0, 0, 30.0),
    (7, 16, [200, 113], [90, 113], 1, 1, 256, 128, 0, 0, 0.0),
    (45, 16, [2000, 725], [600, 300], 1, 1, 128, 128, 0, 0, 0.0),
    (21, 32, [700, 680, 673], [400, 9, 300], 40, 1, 128, 128, 0, 0, 0.0),
]


@pytest.mark.parametrize("entries,page,lens,new,heads,R,D,G,window,sinks,cap", PAST)
def test_keys_past_the_table_are_not_seen(entries, page, lens, new, heads, R, D, G, window, sinks, cap):
    held = [min(n, entries * page) for n in lens]
    c = kv.Cache(held, new, heads, D, G, page, seed=sum(lens) + D, width=entries).fill()
    c.lens = lens
    kv_cases.attend(c, R, single=all(m == 1 for m in new), window=window, sinks=sinks, cap=cap, stored=held)
