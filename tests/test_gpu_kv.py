"""The 4-bit cache of keys and values on the GPU: what tpq_kv_append writes, what tpq_kv_read gives back and
tpq_kv_attention makes of it, against plain implementations (kv_reference)."""
import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2411_07942_amd as tpq
import workloads as wl

pytestmark = pytest.mark.gpu

GARBAGE = 0xFF  # every bf16 of it a NaN


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def bf16_tensor(x):
    """fp32 array of bf16 values -> bf16 tensor on the GPU."""
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.bfloat16).cuda()


class Cache:
    """Sequences of given lengths, n new tokens of each, in pages of a shuffled pool; whatever no token owns is garbage."""

    def __init__(self, lens, new, heads, D, G, page, seed, width=None):
        rng = np.random.default_rng(seed)
        self.lens, self.new, self.heads, self.D, self.G, self.page = lens, new, heads, D, G, page
        used = [-(-n // page) for n in lens]
        self.n_pages = sum(used) + 3
        pool = rng.permutation(self.n_pages)
        self.table = rng.integers(-(1 << 31), (1 << 31) - 1, (len(lens), width or max(max(used), 1) + 1)).astype(np.int32)
        at = 0
        for b, u in enumerate(used):
            self.table[b, :u] = pool[at:at + u]
            at += u
        self.starts = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
        self.rows = int(self.starts[-1])
        self.L = tpq.kv_layout_init(heads, D, G, page)
        self.bytes = np.full(self.n_pages * self.L.page_bytes, GARBAGE, np.uint8)
        self.rng = rng

    def place(self, b, pos):
        pos = np.asarray(pos)
        return self.table[b][pos // self.page], pos % self.page

    def fill(self, spread=1.0, offset=0.0):
        """Keys and values for every token; self.k, self.v: each sequence's values [n, heads, D]."""
        self.k, self.v = [], []
        for b, n in enumerate(self.lens):
            pages, slots = self.place(b, np.arange(n))
            for key, to in ((True, self.k), (False, self.v)):
                x = self.rng.standard_normal((n, self.heads, self.D)).astype(np.float32) * spread + offset
                x[..., :: 17] *= 4.0
                codes, scale, zero = ref.quantise(ref.bf16(x), self.G) if n else (np.zeros((0, self.heads, self.D), np.uint8),) + 2 * (
                    np.zeros((0, self.heads, self.D // self.G), np.uint16),)
                ref.store(self.bytes, self.n_pages, self.D, self.G, self.page, pages, slots, key, codes, scale, zero)
                to.append(ref.values(codes, scale, zero))
        return self

    def batch(self, single=False, max_new=None, max_len=None):
        return tpq.KvBatch(dev(self.table), dev(np.asarray(self.lens, np.int32)), None if single else dev(self.starts),
                           max_new or (1 if single else max(max(self.new), 1)), max_len)


# ---- append and read --------------------------------------------------------------------------------

APPEND = [  # lens, new, heads, q_heads, D, G, page, rot, pairs
    ([1], [1], 1, 1, 128, 128, 16, 128, False),
    ([17, 300, 16, 33], [1, 1, 1, 1], 2, 4, 128, 128, 16, 128, True),
    ([129, 0, 70, 5], [129, 0, 33, 5], 3, 6, 64, 32, 32, 32, False),
    ([40, 260], [39, 7], 1, 5, 256, 256, 16, 256, False),
    ([64, 65, 63], [64, 2, 17], 2, 2, 256, 64, 64, 96, True),
    ([257], [256], 5, 5, 128, 64, 128, 0, False),
    ([300, 299], [100, 1], 2, 3 * 2, 64, 64, 256, 16, True),
]


@pytest.mark.parametrize("lens,new,heads,q_heads,D,G,page,rot,pairs", APPEND)
def test_append_and_read(lens, new, heads, q_heads, D, G, page, rot, pairs):
    c = Cache(lens, new, heads, D, G, page, seed=D + G + page)
    rng, T, spare = c.rng, c.rows, 2
    x = rng.standard_normal((T + spare, q_heads + 2 * heads, D)).astype(np.float32) * 3
    x[..., ::29] *= 30
    x[0, q_heads] = 0.75                     # constant groups; zeros of both signs
    x[0, -1] = np.where(np.arange(D) % 2, 0.0, -0.0)
    x = ref.bf16(x)
    cos, sin = (rng.standard_normal((max(max(lens), 1), rot // 2)).astype(np.float32) for _ in range(2))
    qkv = torch.zeros((T + spare, q_heads + 2 * heads + 1, D), dtype=torch.bfloat16, device="cuda")
    qkv[:, :-1] = bf16_tensor(x)
    q_out = torch.full((T + spare, q_heads * D + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    cache = dev(c.bytes)
    tpq.kv_append(c.L, cache, c.batch(), qkv[:, q_heads:q_heads + heads], qkv[:, q_heads + heads:-1],
                  dev(cos) if rot else None, dev(sin) if rot else None, pairs, qkv[:, :q_heads], q_out[:, :q_heads * D])
    k_out = torch.full((T + spare, heads, D), 7.0, device="cuda")
    v_out = torch.full((T + spare, heads, D), 7.0, device="cuda")
    tpq.kv_read(c.L, cache, c.batch(), k_out, v_out)
    k_half = torch.full((T + spare, heads, D), 7.0, dtype=torch.bfloat16, device="cuda")
    tpq.kv_read(c.L, cache, c.batch(), k_half, None)
    v_only = torch.full((T + spare, heads * D), 7.0, device="cuda")
    tpq.kv_read(c.L, cache, c.batch(), None, v_only)
    torch.cuda.synchronize()

    b = np.repeat(np.arange(len(lens)), new)
    pos = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, new)]).astype(int)
    q, k, v = (x[:T, s] for s in (slice(0, q_heads), slice(q_heads, q_heads + heads), slice(q_heads + heads, None)))
    if rot:
        q, k = ref.rotate(q, cos[pos], sin[pos], pairs), ref.rotate(k, cos[pos], sin[pos], pairs)
    pages, slots = c.table[b, pos // page], pos % page
    for key, y, got in ((True, k, k_out), (False, v, v_out)):
        codes, scale, zero = ref.quantise(np.ascontiguousarray(y), G)
        ref.store(c.bytes, c.n_pages, D, G, page, pages, slots, key, codes, scale, zero)
        want = ref.values(codes, scale, zero)
        assert np.array_equal(got[:T].cpu().numpy().view(np.uint32), want.view(np.uint32))
        if key:
            assert np.array_equal(wl.to_bits(k_half[:T]), ref.bits(ref.bf16(want)))
        else:
            assert np.array_equal(v_only[:T].cpu().numpy().reshape(want.shape), want)
    assert np.array_equal(cache.cpu().numpy(), c.bytes)  # (everything but the new tokens' bytes is as it was)
    assert np.array_equal(wl.to_bits(q_out[:T, :q_heads * D]).reshape(q.shape), ref.bits(q))
    assert (q_out[:, q_heads * D:] == 7.0).all() and (q_out[T:] == 7.0).all()
    for t in (k_out, v_out, k_half, v_only):
        assert (t[T:] == 7.0).all()


@pytest.mark.parametrize("pairs", [False, True])
def test_queries_in_place(pairs):
    c = Cache([50], [20], 1, 128, 64, 16, seed=1)
    x = ref.bf16(c.rng.standard_normal((20, 5, 128)).astype(np.float32))
    cos, sin = (c.rng.standard_normal((50, 64)).astype(np.float32) for _ in range(2))
    q, k = bf16_tensor(x[:, :4]), bf16_tensor(x[:, 4:])
    tpq.kv_append(c.L, dev(c.bytes), c.batch(), k, k, dev(cos), dev(sin), pairs, q)
    assert np.array_equal(wl.to_bits(q), ref.bits(ref.rotate(x[:, :4], cos[30:], sin[30:], pairs)))


def test_append_one_token_each_without_starts():
    """Row b is sequence b's token; a second step goes behind the first one."""
    lens = [1, 16, 31, 200]
    c = Cache([n + 1 for n in lens], [1] * 4, 2, 128, 128, 16, seed=3)
    cache, steps = dev(c.bytes), []
    for step in range(2):
        c.lens = [n + step for n in lens]
        x = ref.bf16(c.rng.standard_normal((4, 2, 2, 128)).astype(np.float32))
        tpq.kv_append(c.L, cache, c.batch(single=True), bf16_tensor(x[:, 0]), bf16_tensor(x[:, 1]))
        pos = np.asarray(c.lens) - 1
        for key in (True, False):
            ref.store(c.bytes, c.n_pages, 128, 128, 16, c.table[np.arange(4), pos // 16], pos % 16, key,
                      *ref.quantise(np.ascontiguousarray(x[:, 0 if key else 1]), 128))
    assert np.array_equal(cache.cpu().numpy(), c.bytes)


def test_absent_tokens_are_neither_written_nor_read():
    """Pages that are none, positions past the table or the rotation's, more new tokens than tokens, starts that are no
    ranges, more new tokens than max_new: the rows concerned stay as they were, the others' are right."""
    lens, new = [40, 20, 20, 10, 33], [40, 20, 4, 10, 33]
    c = Cache(lens, new, 1, 64, 64, 16, seed=5, width=3)
    c.table[0, 1] = c.n_pages                   # tokens 16 .. 31 of sequence 0
    c.table[1, 0] = -1                          # tokens 0 .. 15 of sequence 1
    c.lens[4] = 60                              # tokens 48 .. 59 of sequence 4 lie past its table; its page 2 is unowned
    c.table[4, 2] = c.n_pages - 1
    c.lens[3] = 5                               # 10 new tokens, 5 tokens: the first five have no position
    x = ref.bf16(c.rng.standard_normal((c.rows, 2, 64)).astype(np.float32))
    K, V = bf16_tensor(x[:, :1]), bf16_tensor(x[:, 1:])
    cos = torch.ones((45, 8), device="cuda")    # positions from 45 on have no rotation
    cache, keep = dev(c.bytes), c.rows
    k_out = torch.full((c.rows, 1, 64), 7.0, device="cuda")
    batch = c.batch(max_new=35)                 # tokens 35 .. 39 of sequence 0 are left out
    tpq.kv_append(c.L, cache, batch, K, V, cos, torch.zeros_like(cos))
    tpq.kv_read(c.L, cache, batch, k_out, None)
    good = np.zeros(keep, bool)
    for b in range(5):
        for i in range(min(new[b], 35)):
            p = c.lens[b] - new[b] + i
            if 0 <= p < 45 and p < 48 and 0 <= c.table[b, p // 16] < c.n_pages:
                r = c.starts[b] + i
                good[r] = True
                for key in (True, False):
                    ref.store(c.bytes, c.n_pages, 64, 64, 16, [c.table[b, p // 16]], [p % 16], key, *ref.quantise(x[r:r + 1, 0 if key else 1][:, None], 64))
    assert np.array_equal(cache.cpu().numpy(), c.bytes)
    codes = ref.quantise(np.ascontiguousarray(x[:, :1]), 64)
    assert np.array_equal(k_out.cpu().numpy()[good], ref.values(*codes)[good])
    # tokens 45 .. 47 of sequence 4 exist in the cache, unwritten; all others that were left out are left alone
    seq4 = np.zeros(keep, bool)
    seq4[c.starts[4] + 18:c.starts[4] + 21] = True
    assert (k_out.cpu().numpy()[~good & ~seq4] == 7.0).all()

    for starts in ([-1, 3, 9], [0, 5, 200], [7, 3, 9]):
        c2 = Cache([20, 20], [3, 6], 1, 64, 64, 16, seed=6)
        c2.starts = np.asarray(starts, np.int32)
        cache = dev(c2.bytes)
        tpq.kv_append(c2.L, cache, c2.batch(max_new=20), K[:9], V[:9])
        got = cache.cpu().numpy()
        b, rows = (1, range(3, 9)) if starts[0] in (-1, 7) else (0, range(0, 5))
        for i, r in enumerate(rows):
            p = 20 - len(rows) + i
            for key in (True, False):
                ref.store(c2.bytes, c2.n_pages, 64, 64, 16, [c2.table[b, p // 16]], [p % 16], key, *ref.quantise(x[r:r + 1, 0 if key else 1][:, None], 64))
        assert np.array_equal(got, c2.bytes)


# ---- attention ---------------------------------------------------------------------------------------

def bound(want, reach, mass, wide, D, n, scale, few):
    """What an output may be off: half a bf16 step of it (2^-8), and the weights' error times the values.
    few: codes are exact; weights are pairs of bf16 (half a step twice: 2^-16).  many: keys and values in fp16 at a scale
    of their own (half a step 2^-11 of each element), weights in fp16 (2^-11); below its normal range fp16's steps stay 2^-24, 2^-34 of the
    largest.  Scores in fp32: D products added to 16 at most 143 times a code's step (2^-24 each, twice their number for
    the matrix unit's own order), seen through the exponential by both numerator and sum (hence 2 *).  The accumulators
    add n / 32 times at 143 / 15 of the weights' mass, whose codes reach 15 steps."""
    scores = scale * reach[..., None] * ((0 if few else 2.0 ** -10) + (2 * D + 64) * 10 * 2.0 ** -24) + 2.0 ** -20
    sums = (n / 32 + 64) * 10 * 2.0 ** -24
    return np.abs(want) * 2.0 ** -8 + (2 * scores + (2.0 ** -16 if few else 2.0 ** -10) + sums) * (mass + wide)[..., None]


def run_attention(c, R, single=False, window=0, sinks=0, cap=0.0, scale=None, max_len=None, q_scale=1.0, spare=2, absent=None):
    """The call on the GPU against the reference.  absent(b, keys) -> which keys of a sequence count as absent."""
    D, H = c.D, c.heads
    scale = D ** -0.5 if scale is None else scale
    T = c.rows
    q = ref.bf16(c.rng.standard_normal((T + spare, H * R, D)).astype(np.float32) * q_scale)
    Q = torch.zeros((T + spare, H * R + 1, D), dtype=torch.bfloat16, device="cuda")
    Q[:, :-1] = bf16_tensor(q)
    out = torch.full((T + spare, H * R * D + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    batch = c.batch(single, max_len=max_len)
    ws = tpq.kv_attention_workspace(c.L, batch, H * R, "cuda").fill_(GARBAGE)
    cache = dev(c.bytes)
    tpq.kv_attention(c.L, cache, batch, Q[:, :-1], out[:, :H * R * D], scale, ws, window, sinks, cap)
    torch.cuda.synchronize()
    assert np.array_equal(cache.cpu().numpy(), c.bytes)
    assert (out[:, H * R * D:] == 7.0).all() and (out[T:] == 7.0).all()
    got = out[:T, :H * R * D].float().cpu().numpy().reshape(T, H, R, D)
    few = max(c.new) * R <= 32
    for b, (n, m) in enumerate(zip(c.lens, c.new)):
        if m == 0:
            continue
        pos = np.arange(n - m, n)
        keep = np.ones(n, bool) if absent is None else ~absent(b, np.arange(n))
        rows = slice(int(c.starts[b]), int(c.starts[b]) + m)
        for h in range(H):
            k, v = c.k[b][:n, h].astype(np.float64), c.v[b][:n, h].astype(np.float64)
            want, reach, mass = ref.attention(q[rows, h * R:(h + 1) * R].astype(np.float64), k, v, pos, scale, window, sinks, cap) if keep.all() else \
                attention_without(q[rows, h * R:(h + 1) * R].astype(np.float64), k, v, pos, scale, window, sinks, cap, keep)
            wide = np.abs(v).max() * 2.0 ** -20 if n else 0.0
            lim = bound(want, reach, mass, wide, D, max(n, 1), scale, few)
            err = np.abs(got[rows, h] - want)
            assert np.isfinite(got[rows, h]).all()
            assert (err <= lim).all(), (b, h, float((err - lim).max()), float((err / (lim + 1e-30)).max()))
    return got


def attention_without(q, k, v, pos, scale, window, sinks, cap, keep):
    """As ref.attention, with keys that count as absent."""
    m, R, D = q.shape
    out, reach, mass = np.zeros((m, R, D)), np.zeros((m, R)), np.zeros((m, R))
    for i in range(m):
        seen = np.flatnonzero(ref.visible(pos[i], k.shape[0], window, sinks) & keep)
        if seen.size:
            o, r, w = ref.attention(q[i:i + 1], k[seen], v[seen], np.asarray([seen.size]), scale, 0, 0, cap)
            out[i], reach[i], mass[i] = o[0], r[0], w[0]
    return out, reach, mass


FEW = [  # lens, new, heads, R, D, G, page, window, sinks, cap
    ([1], [1], 1, 1, 128, 128, 16, 0, 0, 0.0),
    ([2, 15, 16, 17, 31, 32, 33], [1] * 7, 2, 1, 128, 128, 16, 0, 0, 0.0),
    ([640, 127, 129, 4000], [1] * 4, 2, 4, 128, 64, 64, 0, 0, 0.0),
    ([1000, 77], [1, 1], 1, 16, 128, 32, 32, 0, 0, 30.0),
    ([513, 300, 31], [1] * 3, 3, 5, 64, 64, 16, 0, 0, 0.0),
    ([513, 300, 31], [1] * 3, 3, 2, 64, 32, 128, 100, 0, 0.0),
    ([700, 90], [1, 1], 2, 3, 256, 256, 16, 0, 0, 0.0),
    ([700, 90], [1, 1], 2, 8, 256, 128, 32, 0, 0, 0.0),
    ([333], [1], 1, 1, 256, 64, 256, 64, 3, 0.0),
    ([200, 5], [1, 1], 1, 9, 256, 32, 16, 0, 0, 10.0),
    ([5000, 4, 64, 65, 66], [1] * 5, 2, 4, 128, 128, 16, 64, 4, 0.0),     # windows that start at a tile, inside one, before the text
    ([2000, 1999, 2031], [1] * 3, 1, 4, 128, 64, 16, 1, 0, 0.0),          # a window of one: the token itself
    ([2000, 90, 20], [1] * 3, 1, 2, 128, 128, 16, 33, 70, 0.0),           # as many first tokens as meet the window
    ([300, 9, 64, 3], [5, 5, 3, 0], 2, 4, 128, 64, 16, 0, 0, 0.0),        # a few tokens each, one sequence without any
    ([300, 6], [6, 6], 1, 5, 64, 32, 32, 50, 2, 20.0),
    ([100, 40], [16, 3], 2, 2, 128, 128, 16, 0, 0, 0.0),
    ([80, 40], [8, 3], 1, 4, 256, 128, 16, 24, 1, 0.0),
]


@pytest.mark.parametrize("lens,new,heads,R,D,G,page,window,sinks,cap", FEW)
def test_attention_of_few_rows(lens, new, heads, R, D, G, page, window, sinks, cap):
    c = Cache(lens, new, heads, D, G, page, seed=sum(lens) + D).fill()
    run_attention(c, R, single=all(m == 1 for m in new), window=window, sinks=sinks, cap=cap)


MANY = [
    ([33], [33], 1, 1, 128, 128, 16, 0, 0, 0.0),
    ([300], [300], 2, 1, 128, 128, 64, 0, 0, 0.0),
    ([500, 37, 200, 1], [129, 37, 1, 1], 2, 4, 128, 64, 16, 0, 0, 0.0),
    ([300, 260], [70, 260], 1, 3, 64, 32, 32, 0, 0, 30.0),
    ([300, 64], [64, 64], 1, 8, 64, 64, 16, 40, 3, 0.0),
    ([400], [257], 1, 2, 256, 256, 16, 0, 0, 0.0),
    ([400, 100], [100, 99], 1, 4, 256, 64, 64, 90, 5, 0.0),
    ([200, 90], [50, 90], 2, 16, 128, 32, 128, 0, 0, 0.0),
    ([1500, 700], [40, 300], 1, 1, 128, 128, 256, 128, 20, 0.0),
    ([700], [640], 1, 1, 256, 32, 32, 1, 0, 0.0),
]


@pytest.mark.parametrize("lens,new,heads,R,D,G,page,window,sinks,cap", MANY)
def test_attention_of_many_rows(lens, new, heads, R, D, G, page, window, sinks, cap):
    c = Cache(lens, new, heads, D, G, page, seed=sum(lens) + D).fill()
    run_attention(c, R, window=window, sinks=sinks, cap=cap)


@pytest.mark.parametrize("new,R", [(1, 1), (1, 4), (9, 4), (50, 2), (150, 1)])
@pytest.mark.parametrize("spread,offset,q_scale", [(1e-4, 0.0, 1e-3), (3e4, 0.0, 1e-5), (1.0, 25.0, 1.0), (1e5, 1e6, 1e-6), (1.0, 0.0, 30.0)])
def test_attention_of_other_ranges(new, R, spread, offset, q_scale):
    """Values far outside fp16's range, with a mean that dwarfs their spread, tiny ones; scores that leave one key."""
    c = Cache([190, 150], [new, new], 1, 128, 64, 16, seed=new).fill(spread, offset)
    run_attention(c, R, single=new == 1, q_scale=q_scale)


@pytest.mark.parametrize("new,R", [(1, 4), (40, 2)])
def test_absent_keys_are_not_seen(new, R):
    c = Cache([190, 150, 64], [new, min(new, 20), new], 2, 128, 128, 32, seed=new).fill()
    c.table[0, 2], c.table[1, 0], c.table[2, :2] = -5, c.n_pages, 1 << 30
    run_attention(c, R, absent=lambda b, j: (j // 32 == 2) if b == 0 else (j // 32 == 0) if b == 1 else j < 64)


@pytest.mark.parametrize("new,R", [(1, 4), (40, 2)])
def test_more_new_tokens_than_tokens_and_empty_sequences(new, R):
    """Rows without a position see nothing and come out 0; so do all rows of a sequence of no tokens."""
    c = Cache([0, 30, 3], [new, new, new], 1, 128, 128, 16, seed=new).fill()
    got = run_attention(c, R)
    assert (got[:new] == 0).all()


@pytest.mark.parametrize("new,R", [(1, 2), (60, 1)])
def test_garbage_in_hidden_keys(new, R):
    """NaN and infinities among keys that lie before the window."""
    c = Cache([250], [new], 1, 128, 64, 16, seed=new).fill()
    cells = c.bytes.reshape(c.n_pages, 1, -1)
    for j in range(4, 250 - new - 40):
        p, s = c.place(0, j)
        meta = cells[p, 0, 16 * 128:].view(np.uint16).reshape(2, 2, 16, 2)
        meta[:, :, s, 0], meta[:, :, s, 1] = (0x7F80, 0xFF80) if j % 2 else (0x7FC0, 0x7F80)
    run_attention(c, R, window=40, sinks=3)


@pytest.mark.parametrize("new", [1, 3, 100])
def test_attention_is_the_same_again_and_by_other_splits(new):
    """Twice the same bits; another hint of the length, and so other splits, within the bound."""
    c = Cache([3000, 500], [new, new], 2, 128, 128, 16, seed=9).fill()
    state = c.rng.bit_generator.state
    first = run_attention(c, 2)
    for max_len in (None, 16, 600, 3000):
        c.rng.bit_generator.state = state
        again = run_attention(c, 2, max_len=max_len)
        if max_len is None:
            assert np.array_equal(first, again)


def test_long_cache_past_4_gib():
    """Page numbers whose bytes lie past 2^32, in a pool with room for them."""
    L = tpq.kv_layout_init(8, 128, 128, 64)
    n_pages = (1 << 32) // L.page_bytes + 64
    cache = torch.zeros(n_pages * L.page_bytes, dtype=torch.uint8, device="cuda")
    lens = dev(np.asarray([200, 150], np.int32))
    table = dev(np.asarray([[n_pages - 1, 3, n_pages - 7, n_pages - 2], [n_pages - 3, 1, n_pages - 5, 0]], np.int32))
    small = dev(np.asarray([[0, 1, 2, 3], [4, 5, 6, 7]], np.int32))
    starts = dev(np.asarray([0, 200, 350], np.int32))
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((350, 16, 128), generator=g, device="cuda").to(torch.bfloat16)
    got = []
    for t, pool in ((table, cache), (small, torch.zeros(8 * L.page_bytes, dtype=torch.uint8, device="cuda"))):
        batch = tpq.KvBatch(t, lens, starts, max_new=200)
        tpq.kv_append(L, pool, batch, x[:, :8], x[:, 8:])
        k, v = torch.zeros((350, 8, 128), device="cuda"), torch.zeros((350, 8, 128), device="cuda")
        tpq.kv_read(L, pool, batch, k, v)
        outs = [k, v]
        for b, rows in ((batch, 350), (tpq.KvBatch(t, lens), 2)):
            o = torch.zeros((rows, 16, 128), dtype=torch.bfloat16, device="cuda")
            tpq.kv_attention(L, pool, b, x[:rows], o, 0.1, tpq.kv_attention_workspace(L, b, 16, "cuda"))
            outs.append(o)
        got.append(outs)
        tpq.kv_check(L, pool, batch, 350)
    for a, b in zip(*got):
        assert torch.equal(a, b) and a.abs().sum() > 0


def test_check_reports():
    c = Cache([40, 20], [3, 2], 1, 64, 64, 16, seed=2)
    cache = dev(c.bytes)

    def code(rows=5, **changes):
        d = Cache([40, 20], [3, 2], 1, 64, 64, 16, seed=2)
        for k, v in changes.items():
            if k == "page":
                d.table[v] = d.n_pages
            else:
                setattr(d, k, v)
        try:
            tpq.kv_check(d.L, cache, d.batch(max_new=3), rows)
        except tpq.TpqError as e:
            return e.code
        return tpq.OK
    assert code() == tpq.OK
    assert code(page=(0, 3)) == tpq.OK                       # past the sequence's last token
    assert code(page=(0, 2)) == tpq.ERR_INDEX
    assert code(rows=4) == tpq.ERR_INDEX
    assert code(lens=[2, 20]) == tpq.ERR_INDEX               # fewer tokens than new ones
    assert code(lens=[-1, 20]) == tpq.ERR_INDEX
    assert code(lens=[40, 65]) == tpq.ERR_INDEX              # past the table
    assert code(starts=np.asarray([0, 4, 5], np.int32)) == tpq.ERR_INDEX
    assert code(starts=np.asarray([3, 2, 5], np.int32)) == tpq.ERR_INDEX


# ---- as they are used together -------------------------------------------------------------------------

def test_attention_block_on_one_device():
    """A prompt and then single tokens, captured once and replayed with new lengths: append, attention, the row-parallel
    linear layer with the compression in its epilogue, the exchange's sum.  Every replay against the calls made eagerly, on another stream too."""
    H, R, D, page, B = 2, 2, 128, 16, 3
    E, K = 512, H * R * D
    L = tpq.kv_layout_init(H, D, 64, page)
    g = torch.Generator(device="cuda").manual_seed(11)

    def rnd(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)
    LE = tpq.layout_init(E, 8, 128)
    plan = tpq.plan_build(LE, torch.arange(8, dtype=torch.int32, device="cuda") * 5)
    Wp = tpq.gemm_weights(LE, plan, rnd(E, K) * 0.05)
    cos, sin = torch.rand((64, 64), generator=g, device="cuda"), torch.rand((64, 64), generator=g, device="cuda")
    table = torch.randperm(24, generator=g, device="cuda", dtype=torch.int32)[:12].view(B, 4).contiguous()
    prompt = [13, 1, 30]
    starts = torch.tensor([0, 13, 14, 44], dtype=torch.int32, device="cuda")

    def begin():
        cache = tpq.kv_cache(L, 24, "cuda").fill_(GARBAGE)
        lens = torch.tensor(prompt, dtype=torch.int32, device="cuda")
        return cache, lens
    first = rnd(44, H * R + 2 * H, D)
    steps = [rnd(B, H * R + 2 * H, D) for _ in range(4)]

    def prefill(cache, lens):
        batch = tpq.KvBatch(table, lens, starts, max_new=30)
        q, o = torch.empty((44, H * R, D), dtype=torch.bfloat16, device="cuda"), torch.empty((44, H * R, D), dtype=torch.bfloat16, device="cuda")
        tpq.kv_append(L, cache, batch, first[:, H * R:H * R + H], first[:, H * R + H:], cos, sin, False, first[:, :H * R], q)
        tpq.kv_attention(L, cache, batch, q, o, D ** -0.5, tpq.kv_attention_workspace(L, batch, H * R, "cuda"))
        return o

    class Step:
        def __init__(self, cache, lens):
            self.x = torch.empty((B, H * R + 2 * H, D), dtype=torch.bfloat16, device="cuda")
            self.q, self.o = (torch.empty((B, H * R, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            self.msg, self.out = tpq.Message(LE, B, "cuda"), torch.empty((B, E), dtype=torch.bfloat16, device="cuda")
            self.lens, self.batch = lens, tpq.KvBatch(table, lens)
            self.ws = tpq.kv_attention_workspace(L, self.batch, H * R, "cuda")
            x = self.x
            self.calls = [
                tpq.kv_append_call(L, cache, self.batch, x[:, H * R:H * R + H], x[:, H * R + H:], cos, sin, False, x[:, :H * R], self.q),
                tpq.kv_attention_call(L, cache, self.batch, self.q, self.o, D ** -0.5, self.ws),
                tpq.gemm_encode_call(LE, self.o.view(B, K), Wp, self.msg),
                tpq.decode_reduce_call(LE, plan, [self.msg], self.out, tpq.ACC_FP32)]

        def __call__(self, stream=None):
            for c in self.calls:
                c(stream)

    def run(graph, stream=None):
        cache, lens = begin()
        outs = [prefill(cache, lens).clone()]
        step = Step(cache, lens)
        torch.cuda.synchronize()
        if graph:
            step.x.copy_(steps[0])
            lens += 1
            step()                              # (warm; the same token again by the first replay)
            lens -= 1
            torch.cuda.synchronize()
            gr = torch.cuda.CUDAGraph()
            with torch.cuda.graph(gr):
                step()
        for x in steps:
            step.x.copy_(x)
            lens += 1
            if graph:
                gr.replay()
            elif stream is not None:
                stream.wait_stream(torch.cuda.current_stream())
                step(stream)
                torch.cuda.current_stream().wait_stream(stream)
            else:
                step()
            outs += [step.o.clone(), step.out.clone()]
            torch.cuda.synchronize()
        return outs, cache.cpu()
    eager, cache0 = run(False)
    for graph, stream in ((True, None), (False, torch.cuda.Stream())):
        outs, cache1 = run(graph, stream)
        assert all(torch.equal(a, b) for a, b in zip(eager, outs)) and torch.equal(cache0, cache1)
    assert all(torch.isfinite(o.float()).all() for o in eager)
    # the last step against the definition
    vis = [n + len(steps) for n in prompt]
    batch = tpq.KvBatch(table, torch.tensor(vis, dtype=torch.int32, device="cuda"),
                        torch.tensor(np.concatenate(([0], np.cumsum(vis))), dtype=torch.int32, device="cuda"), max_new=max(vis))
    k, v = torch.empty((sum(vis), H, D), device="cuda"), torch.empty((sum(vis), H, D), device="cuda")
    tpq.kv_read(L, cache0.cuda(), batch, k, v)
    k, v = k.cpu().numpy().astype(np.float64), v.cpu().numpy().astype(np.float64)
    q = ref.rotate(steps[-1][:, :H * R].float().cpu().numpy(), cos.cpu().numpy()[np.asarray(vis) - 1], sin.cpu().numpy()[np.asarray(vis) - 1], False)
    at = np.concatenate(([0], np.cumsum(vis)))
    for b in range(B):
        for h in range(H):
            want, reach, mass = ref.attention(q[b:b + 1, h * R:(h + 1) * R].astype(np.float64), k[at[b]:at[b + 1], h], v[at[b]:at[b + 1], h],
                                              [vis[b] - 1], D ** -0.5)
            got = eager[-2][b].float().cpu().numpy().reshape(H, R, D)[h]
            assert (np.abs(got - want[0]) <= bound(want, reach, mass, 0.0, D, vis[b], D ** -0.5, True)[0]).all()
