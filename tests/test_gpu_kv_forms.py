"""The 4-bit cache of keys and values on the GPU in the forms that only some batches take: many sequences, one long one among
short ones, columns by group, tiles of 32 and of 256 rows, large calls of append and read."""
import numpy as np
import pytest
import torch

import paper_2411_07942_amd as tpq
import test_gpu_kv as kv

pytestmark = pytest.mark.gpu


def lengths(count, lo, hi, seed):
    return [int(n) for n in np.random.default_rng(seed).integers(lo, hi + 1, count)]


# heads of 128 and 64 in four units a lane (31 + 31 + 31 units leave a rest of one); more than 64 and more than 4096 sequences,
# runs of sequences without new tokens among them
APPEND = [  # lens, new, heads, q_heads, D, G, page, rot, pairs
    ([1500, 700, 0, 30], [1400, 690, 0, 13], 31, 31, 128, 64, 16, 128, False),
    ([1200, 901, 9], [1200, 900, 1], 31, 31, 64, 32, 64, 32, True),
    ([420, 200], [409, 195], 31, 31, 256, 32, 16, 256, False),
    (lengths(130, 4, 60, 1), lengths(130, 0, 3, 2), 2, 2, 128, 128, 16, 64, False),
    ([n + 1 for n in lengths(5000, 0, 20, 3)], [1] * 70 + [0] * 300 + lengths(4630, 0, 1, 4), 1, 1, 64, 64, 16, 64, True),
]


@pytest.mark.parametrize("case", range(len(APPEND)))
def test_append_and_read(case):
    kv.test_append_and_read(*APPEND[case])


FEW = [  # lens, new, heads, R, D, G, page, window, sinks, cap
    # a column for each row and group: one tile, two tiles, all rows of a head of 256
    ([3000, 31, 700], [1, 1, 1], 2, 4, 128, 32, 32, 0, 0, 0.0),
    ([900, 17], [1, 1], 2, 3, 128, 32, 16, 100, 4, 30.0),
    ([900, 64], [1, 1], 2, 7, 128, 32, 16, 0, 0, 0.0),
    ([900, 33], [1, 1], 2, 8, 128, 64, 16, 64, 2, 0.0),
    ([900, 33], [1, 1], 2, 8, 64, 32, 128, 0, 0, 0.0),
    ([1100, 5], [1, 1], 2, 4, 256, 64, 16, 0, 0, 0.0),
    ([1100, 5], [1, 1], 1, 15, 256, 64, 16, 0, 0, 20.0),
    ([1100, 48], [4, 3], 1, 8, 256, 64, 16, 300, 3, 0.0),
    ([1100, 48], [1, 1], 2, 2, 256, 32, 16, 0, 0, 0.0),
    ([1100, 48], [2, 2], 1, 4, 256, 32, 16, 200, 40, 0.0),
    ([600, 90], [3, 1], 2, 2, 128, 32, 16, 0, 0, 0.0),
    # 32 rows a tile
    ([900, 40], [1, 1], 2, 20, 128, 128, 16, 0, 0, 0.0),
    ([900, 40], [8, 5], 1, 4, 64, 64, 16, 100, 3, 0.0),
    ([333, 20], [31, 20], 1, 1, 64, 64, 256, 0, 0, 10.0),
]


@pytest.mark.parametrize("lens,new,heads,R,D,G,page,window,sinks,cap", FEW)
def test_attention_of_few_rows(lens, new, heads, R, D, G, page, window, sinks, cap):
    c = kv.Cache(lens, new, heads, D, G, page, seed=sum(lens) + D).fill()
    kv.run_attention(c, R, single=all(m == 1 for m in new), window=window, sinks=sinks, cap=cap)


LISTED = [  # lens, new, heads, R, D, G, page, window
    # more tiles of rows than the device takes at once, and a long sequence among short ones
    ([300] * 40 + [9000] + lengths(60, 0, 400, 5), [1] * 101, 8, 1, 128, 128, 64, 0),
    # more than 64 sequences, some without new tokens, some cut
    (lengths(70, 5, 900, 6), lengths(70, 0, 4, 7), 2, 4, 128, 128, 16, 0),
    (lengths(150, 3, 500, 8), lengths(150, 0, 3, 9), 1, 8, 64, 64, 32, 0),
    (lengths(67, 3, 2500, 10), [1] * 67, 1, 2, 256, 64, 32, 700),
    # many rows: cut sequences of unlike lengths, and more than 64 of them
    ([3100, 1700], [70, 33], 2, 1, 128, 128, 16, 0),
    ([2100, 600, 40], [40, 37, 40], 1, 2, 256, 128, 16, 0),
    ([3000, 2800], [34, 50], 1, 1, 64, 32, 64, 1500),
    (lengths(75, 40, 600, 11), lengths(75, 0, 40, 12), 1, 2, 128, 64, 16, 0),
    ([3000, 2800], [70, 66], 1, 1, 64, 32, 64, 1500),
    # more than 4096 sequences: a long one among them; two tiles of rows, none cut
    ([n for n in lengths(2500, 0, 20, 13)] + [9000] + lengths(2600, 0, 20, 14), [1] * 5101, 1, 1, 64, 64, 16, 0),
    ([n + 2 for n in lengths(4200, 0, 20, 15)], lengths(4200, 0, 2, 16), 1, 16, 64, 64, 16, 0),
    # tiles of 16 rows, up to 64 of them
    ([900, 2000, 40], [64, 1, 40], 2, 1, 128, 128, 16, 0),
    ([900, 2000, 40], [15, 16, 9], 1, 4, 256, 128, 32, 500),
    ([64, 50], [64, 50], 3, 1, 64, 64, 16, 0),
]


@pytest.mark.parametrize("case", range(len(LISTED)))
def test_attention_over_a_list_of_sequences(case):
    lens, new, heads, R, D, G, page, window = LISTED[case]
    c = kv.Cache(lens, new, heads, D, G, page, seed=case + 50).fill()
    kv.run_attention(c, R, single=all(m == 1 for m in new), window=window, sinks=2 if window else 0)


@pytest.mark.parametrize("lens,new,heads,D,G,window", [
    ([700], [512], 128, 64, 32, 0),
    ([600, 650], [600, 520], 64, 64, 64, 90),
    ([760], [700], 86, 128, 128, 0),
    ([700], [690], 86, 128, 32, 200),
])
def test_attention_of_256_rows_a_tile(lens, new, heads, D, G, window):
    c = kv.Cache(lens, new, heads, D, G, 64, seed=heads).fill()
    kv.run_attention(c, 1, window=window, sinks=3 if window else 0)


@pytest.mark.parametrize("lens,new,R", [([500, 2000], [1, 1], 4), ([500, 900], [40, 60], 2)])
def test_rows_behind_the_last_sequence(lens, new, R):
    """Matrices with room for far more rows than the batch has, with the workspace of the batch."""
    c = kv.Cache(lens, new, 2, 128, 128, 16, seed=R).fill()
    kv.run_attention(c, R, spare=5000)


def test_a_shorter_hint_than_the_sequences():
    """max_len is a hint: sequences far past it come out as well, in a batch as alone."""
    c = kv.Cache([3000, 200, 2500], [1, 1, 1], 2, 128, 128, 16, seed=8).fill()
    for max_len in (1, 300):
        kv.run_attention(c, 2, single=True, max_len=max_len)


@pytest.mark.parametrize("new", [1, 60])
def test_two_streams_at_once(new):
    """Calls with workspaces of their own on two streams, over one cache: each as alone."""
    c = kv.Cache([900, 700], [new, new], 2, 128, 64, 16, seed=new).fill()
    cache, batch = kv.dev(c.bytes), c.batch(single=new == 1)
    Q = torch.randn((c.rows, 4, 128), device="cuda").to(torch.bfloat16)
    want = torch.empty_like(Q)
    tpq.kv_attention(c.L, cache, batch, Q, want, 0.1, tpq.kv_attention_workspace(c.L, batch, 4, "cuda"))
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros_like(Q) for _ in streams]
    spaces = [tpq.kv_attention_workspace(c.L, batch, 4, "cuda") for _ in streams]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, o, ws in zip(streams, outs, spaces):
            tpq.kv_attention(c.L, cache, batch, Q, o, 0.1, ws, stream=s)
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, want)


@pytest.mark.parametrize("count,new,heads", [(70, 1, 8), (70, 3, 2), (3, 80, 2), (80, 70, 1), (1, 300, 2)])
def test_captured_and_replayed_with_other_lengths(count, new, heads):
    """The list of items, the shares and their sums follow lengths and starts that change between replays; eager work lies between."""
    c = kv.Cache([1500 if b == 1 or count == 1 else 500 for b in range(count)], [new] * count, heads, 128, 128, 16, seed=count, width=1251).fill()
    cache, batch = kv.dev(c.bytes), c.batch(single=new == 1, max_len=20000 if count == 70 else None)
    Q = torch.randn((c.rows, 2 * heads, 128), device="cuda").to(torch.bfloat16)
    out, want = torch.zeros_like(Q), torch.zeros_like(Q)
    ws, ws2 = (tpq.kv_attention_workspace(c.L, batch, 2 * heads, "cuda") for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tpq.kv_attention(c.L, cache, batch, Q, out, 0.1, ws)
    rng = np.random.default_rng(count + new)
    for _ in range(5):
        lens = [int(rng.integers(0, n + 1)) for n in c.lens]
        mine = [int(min(n, rng.integers(0, new + 1))) for n in lens] if new > 1 else [1] * count
        batch.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        if new > 1:
            batch.starts.copy_(torch.tensor(np.concatenate(([0], np.cumsum(mine))), dtype=torch.int32))
        out.fill_(3.0)
        want.fill_(3.0)
        tpq.kv_attention(c.L, cache, batch, Q, want, 0.1, ws2.fill_(kv.GARBAGE))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
