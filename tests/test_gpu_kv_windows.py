"""Attention over the 4-bit cache with a window where a sequence's last tile of rows goes through fewer steps than an earlier one, and
sequences are cut into shares; and calls of 33 to 64 rows, or of 8 groups, at the bound of the kernel that they go to."""
import numpy as np
import pytest
import torch

import kv_cases
import paper_2411_07942_amd as tpq
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


@pytest.mark.parametrize("count,new,heads,R", [(1, 9, 2, 2), (4, 9, 2, 2), (70, 9, 1, 2), (1, 140, 2, 1), (5, 140, 1, 2)])
def test_captured_windows_follow_the_lengths(count, new, heads, R):
    """A captured call over cut, windowed tiles, replayed with other lengths and starts, its workspace full of NaN; eager work between."""
    c = kv.Cache([4000 if b == 0 else 2500 for b in range(count)], [new] * count, heads, 128, 128, 16, seed=count).fill()
    cache, batch = kv.dev(c.bytes), c.batch()
    Q = torch.randn((c.rows, R * heads, 128), device="cuda").to(torch.bfloat16)
    out, want = torch.zeros_like(Q), torch.zeros_like(Q)
    ws, ws2 = (tpq.kv_attention_workspace(c.L, batch, R * heads, "cuda") for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tpq.kv_attention(c.L, cache, batch, Q, out, 0.1, ws, 1000, 3)
    rng = np.random.default_rng(count + new)
    for _ in range(5):
        lens = [int(rng.integers(0, n + 1)) for n in c.lens]
        mine = [int(min(n, rng.integers(0, new + 1))) for n in lens]
        batch.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        batch.starts.copy_(torch.tensor(np.concatenate(([0], np.cumsum(mine))), dtype=torch.int32))
        out.fill_(3.0)
        want.fill_(3.0)
        tpq.kv_attention(c.L, cache, batch, Q, want, 0.1, ws2.fill_(kv.GARBAGE), 1000, 3)
        ws.fill_(kv.GARBAGE)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.isfinite(want.float()).all()
        assert (out[sum(mine):] == 3.0).all()
