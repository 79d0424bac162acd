"""The 4-bit cache of keys and values without a GPU: layout arithmetic, refusals (all before anything is enqueued, so that the
made-up pointers are never followed), and the tests' own reference held against its definitions."""
import ctypes
import math

import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2411_07942_amd as tpq
import workloads as wl


def _p(i=1):
    return ctypes.c_void_p(0x100000 * i)


@pytest.mark.parametrize("heads,D,G,page", [(1, 64, 32, 16), (5, 128, 128, 64), (8, 128, 32, 256), (256, 256, 256, 128)])
def test_layout(heads, D, G, page):
    """8 bytes of scale and zero per token and group beside 4 bits a value, keys and values together."""
    L = tpq.kv_layout_init(heads, D, G, page)
    assert (L.heads, L.D, L.G, L.page, L.ng) == (heads, D, G, page, D // G)
    assert L.cell_bytes == page * (2 * D // 2 + 2 * 4 * (D // G)) and L.page_bytes == heads * L.cell_bytes
    assert L.cell_bytes % 16 == 0 and ctypes.sizeof(L) == 40


@pytest.mark.parametrize("args,code", [
    ((1, 96, 32, 16), tpq.ERR_UNSUPPORTED), ((1, 32, 32, 16), tpq.ERR_UNSUPPORTED), ((1, 512, 128, 16), tpq.ERR_UNSUPPORTED),
    ((1, 64, 128, 16), tpq.ERR_UNSUPPORTED), ((1, 128, 16, 16), tpq.ERR_UNSUPPORTED), ((1, 128, 48, 16), tpq.ERR_UNSUPPORTED),
    ((1, 128, 128, 8), tpq.ERR_UNSUPPORTED), ((1, 128, 128, 48), tpq.ERR_UNSUPPORTED), ((1, 128, 128, 512), tpq.ERR_UNSUPPORTED),
    ((0, 128, 128, 16), tpq.ERR_SHAPE), ((257, 128, 128, 16), tpq.ERR_SHAPE), ((1, 0, 0, 0), tpq.ERR_UNSUPPORTED), ((1, -128, 32, 16), tpq.ERR_UNSUPPORTED),
])
def test_layout_refusals(args, code):
    with pytest.raises(tpq.TpqError) as e:
        tpq.kv_layout_init(*args)
    assert e.value.code == code


def _layout(**kw):
    L = tpq.kv_layout_init(2, 128, 64, 16)
    for k, v in kw.items():
        setattr(L, k, v)
    return L


def _batch(**kw):
    b = tpq._KvBatch(_p(10), _p(11), _p(12), 4, 8, 5, 100, 20, 64, 0)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


BATCHES = [
    (dict(table=None), tpq.ERR_NULL), (dict(lens=None), tpq.ERR_NULL), (dict(table=0x1002), tpq.ERR_ALIGN), (dict(lens=0x1001), tpq.ERR_ALIGN),
    (dict(starts=0x1002), tpq.ERR_ALIGN), (dict(n_seqs=0), tpq.ERR_SHAPE), (dict(n_seqs=65536), tpq.ERR_SHAPE), (dict(ld_table=0), tpq.ERR_SHAPE),
    (dict(ld_table=(1 << 24) + 1), tpq.ERR_SHAPE), (dict(max_new=0), tpq.ERR_SHAPE), (dict(max_new=(1 << 20) + 1), tpq.ERR_SHAPE),
    (dict(max_len=0), tpq.ERR_SHAPE), (dict(max_len=129), tpq.ERR_SHAPE), (dict(rows=-1), tpq.ERR_SHAPE), (dict(rows=1 << 31), tpq.ERR_SHAPE),
    (dict(n_pages=0), tpq.ERR_SHAPE), (dict(n_pages=1 << 31), tpq.ERR_SHAPE),
    (dict(starts=None), tpq.ERR_SHAPE),                       # without starts: one new token
    (dict(starts=None, max_new=1, rows=3), tpq.ERR_SHAPE),    # ... and a row for each
]
LAYOUTS = [(dict(D=96), tpq.ERR_UNSUPPORTED), (dict(G=16), tpq.ERR_UNSUPPORTED), (dict(page=24), tpq.ERR_UNSUPPORTED), (dict(heads=0), tpq.ERR_SHAPE),
           (dict(ng=4), tpq.ERR_SHAPE), (dict(cell_bytes=16), tpq.ERR_SHAPE), (dict(page_bytes=16), tpq.ERR_SHAPE)]


def _calls():
    lib = tpq._load()

    def append(L, b, cache=_p(1), K=_p(2), ldK=256, V=_p(3), ldV=256, cos=_p(4), sin=_p(5), rot=128, rows=100, mode=0, Q=_p(6), ldQ=512, qh=4, Qo=_p(7),
               ldQo=512):
        return lib.tpq_kv_append(L, cache, b, K, ldK, V, ldV, cos, sin, rot, rows, mode, Q, ldQ, qh, Qo, ldQo, None)

    def read(L, b, cache=_p(1), dtype=tpq.OUT_FP32, K=_p(2), ldK=256, V=_p(3), ldV=256):
        return lib.tpq_kv_read(L, cache, b, dtype, K, ldK, V, ldV, None)

    def attention(L, b, cache=_p(1), Q=_p(2), ldQ=512, qh=4, scale=0.1, window=0, sinks=0, cap=0.0, out=_p(3), ldOut=512, ws=_p(4), ws_bytes=1 << 40):
        return lib.tpq_kv_attention(L, cache, b, Q, ldQ, qh, scale, window, sinks, cap, out, ldOut, ws, ws_bytes, None)

    def check(L, b):
        return lib.tpq_kv_check(L, b, None)
    return append, read, attention, check


def _ref(s):
    return None if s is None else ctypes.byref(s)


@pytest.mark.parametrize("which", range(4))
def test_batch_and_layout_refusals(which):
    call = _calls()[which]
    assert call(None, _ref(_batch())) == tpq.ERR_NULL
    assert call(_ref(_layout()), None) == tpq.ERR_NULL
    for kw, code in BATCHES:
        assert call(_ref(_layout()), _ref(_batch(**kw))) == code, kw
    for kw, code in LAYOUTS:
        assert call(_ref(_layout(**kw)), _ref(_batch())) == code, kw
    lib = tpq._load()
    for kw, _ in BATCHES:
        assert lib.tpq_kv_attention_workspace_bytes(_ref(_layout()), _ref(_batch(**kw)), 4) == 0
    for q_heads in (0, 1, 3, 2050, -2):
        assert lib.tpq_kv_attention_workspace_bytes(_ref(_layout()), _ref(_batch()), q_heads) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(cache=None), tpq.ERR_NULL), (dict(K=None), tpq.ERR_NULL), (dict(V=None), tpq.ERR_NULL), (dict(cos=None), tpq.ERR_NULL),
    (dict(sin=None), tpq.ERR_NULL), (dict(Qo=None), tpq.ERR_NULL), (dict(cache=ctypes.c_void_p(0x1008)), tpq.ERR_ALIGN),
    (dict(K=ctypes.c_void_p(0x1008)), tpq.ERR_ALIGN), (dict(V=ctypes.c_void_p(0x1002)), tpq.ERR_ALIGN), (dict(Q=ctypes.c_void_p(0x1008)), tpq.ERR_ALIGN),
    (dict(Qo=ctypes.c_void_p(0x1008)), tpq.ERR_ALIGN), (dict(cos=ctypes.c_void_p(0x1004)), tpq.ERR_ALIGN), (dict(ldK=255), tpq.ERR_SHAPE),
    (dict(ldV=128), tpq.ERR_SHAPE), (dict(ldQ=511), tpq.ERR_SHAPE), (dict(ldQo=256), tpq.ERR_SHAPE), (dict(ldK=260), tpq.ERR_ALIGN),
    (dict(ldV=257), tpq.ERR_ALIGN), (dict(ldQ=516), tpq.ERR_ALIGN), (dict(ldQo=516), tpq.ERR_ALIGN), (dict(rot=-16), tpq.ERR_SHAPE),
    (dict(rot=144), tpq.ERR_SHAPE), (dict(rot=24), tpq.ERR_SHAPE), (dict(rows=0), tpq.ERR_SHAPE), (dict(mode=2), tpq.ERR_UNSUPPORTED),
    (dict(qh=3), tpq.ERR_SHAPE), (dict(qh=0), tpq.ERR_SHAPE), (dict(qh=2048, ldQ=1 << 20, ldQo=1 << 20), tpq.ERR_SHAPE),
])
def test_append_refusals(kw, code):
    assert _calls()[0](_ref(_layout()), _ref(_batch()), **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(cache=None), tpq.ERR_NULL), (dict(dtype=2), tpq.ERR_UNSUPPORTED), (dict(ldK=128), tpq.ERR_SHAPE), (dict(ldV=255), tpq.ERR_SHAPE),
    (dict(ldK=258), tpq.ERR_ALIGN), (dict(ldV=260, dtype=tpq.OUT_BF16), tpq.ERR_ALIGN), (dict(K=ctypes.c_void_p(0x1008)), tpq.ERR_ALIGN),
    (dict(cache=ctypes.c_void_p(0x1004)), tpq.ERR_ALIGN), (dict(K=None, V=None), tpq.OK),
])
def test_read_refusals(kw, code):
    assert _calls()[1](_ref(_layout()), _ref(_batch()), **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(qh=3), tpq.ERR_SHAPE), (dict(qh=0), tpq.ERR_SHAPE), (dict(ldQ=511), tpq.ERR_SHAPE), (dict(ldOut=256), tpq.ERR_SHAPE),
    (dict(ldQ=516), tpq.ERR_ALIGN), (dict(ldOut=516), tpq.ERR_ALIGN), (dict(window=-1), tpq.ERR_SHAPE), (dict(sinks=-1), tpq.ERR_SHAPE),
    (dict(window=(1 << 28) + 1), tpq.ERR_SHAPE), (dict(sinks=(1 << 28) + 1), tpq.ERR_SHAPE), (dict(scale=math.nan), tpq.ERR_SHAPE),
    (dict(scale=math.inf), tpq.ERR_SHAPE), (dict(cap=-1.0), tpq.ERR_SHAPE), (dict(cap=math.inf), tpq.ERR_SHAPE), (dict(cap=math.nan), tpq.ERR_SHAPE),
    (dict(cache=None), tpq.ERR_NULL), (dict(Q=None), tpq.ERR_NULL), (dict(out=None), tpq.ERR_NULL), (dict(ws=None), tpq.ERR_NULL),
    (dict(Q=ctypes.c_void_p(0x1008)), tpq.ERR_ALIGN), (dict(out=ctypes.c_void_p(0x1008)), tpq.ERR_ALIGN), (dict(ws=ctypes.c_void_p(0x1008)), tpq.ERR_ALIGN),
    (dict(cache=ctypes.c_void_p(0x1008)), tpq.ERR_ALIGN),
])
def test_attention_refusals(kw, code):
    assert _calls()[2](_ref(_layout()), _ref(_batch()), **kw) == code


def test_no_rows_is_a_no_op():
    append, read, attention, _ = _calls()
    for call in (append, read, attention):
        assert call(_ref(_layout()), _ref(_batch(rows=0)), cache=None) == tpq.OK


def test_batch_objects_refuse():
    i = torch.zeros((2, 3), dtype=torch.int32)
    with pytest.raises(AssertionError):          # not on a GPU
        tpq.KvBatch(i, i[:, 0].contiguous())


def test_calls_refuse_tensors_that_are_not_on_the_gpu():
    class Fake:  # as a KvBatch on device 0
        _c = tpq._KvBatch(0x1000, 0x1000, None, 2, 3, 1, 0, 0, 0, 0)
    L = tpq.kv_layout_init(1, 64, 64, 16)
    x = torch.zeros((2, 1, 64), dtype=torch.bfloat16)
    cache = torch.zeros(4 * L.page_bytes, dtype=torch.uint8)
    for f, args in ((tpq.kv_append, (x, x)), (tpq.kv_read, (x, x)), (tpq.kv_attention, (x, x, 1.0, cache))):
        with pytest.raises((AssertionError, RuntimeError)):
            f(L, cache, Fake(), *args)
        with pytest.raises((TypeError, AttributeError)):
            f(tpq.layout_init(64, 0, 32), cache, Fake(), *args)
        with pytest.raises((TypeError, AttributeError)):
            f(L, cache, None, *args)


# ---- the reference itself ---------------------------------------------------------------------------

@pytest.mark.parametrize("D", [64, 128, 256])
def test_reference_byte_order(D):
    """Every nibble of a row belongs to one feature, and the orders are those of the header: keys 32 kk + 8 g + j in dword
    g D/32 + kk, 2t in bits 4t, 2t + 1 in bits 16 + 4t; values 16 n + m in bits 4n of chunk m."""
    for key in (True, False):
        assert sorted(ref.nibble_of(D, key)) == list(range(D))
    codes = np.arange(D).astype(np.uint8) % 16
    words = ref.row_bytes(codes, True).view(np.uint32)
    chunks = ref.row_bytes(codes[::-1].copy(), False).reshape(16, D // 32)
    for d in range(D):
        kk, g, j = d // 32, d // 8 % 4, d % 8
        assert (words[g * (D // 32) + kk] >> (4 * (j // 2) + 16 * (j % 2))) & 15 == codes[d]
        n, m = d // 16, d % 16
        assert (chunks[m, n // 2] >> (4 * (n % 2))) & 15 == codes[D - 1 - d]


def test_reference_quantiser_and_rotation():
    """Against one value at a time in 64 bits."""
    rng = np.random.default_rng(0)
    x = ref.bf16(rng.standard_normal((3, 2, 64)).astype(np.float32))
    codes, scale, zero = ref.quantise(x, 32)
    back = ref.values(codes, scale, zero)
    step = wl.bits_to_f32(scale)
    assert (codes <= 15).all() and codes.max() == 15 and codes.min() == 0
    # half a step, the bf16 scale's own rounding (15 steps of 2^-8) and fp32's
    assert (np.abs(back - x) <= np.repeat(step, 32, -1) * (0.5 + 15 * 2.0 ** -8 + 1e-5)).all()
    cos, sin = np.cos(np.arange(3 * 16).reshape(3, 16)).astype(np.float32), np.sin(np.arange(3 * 16).reshape(3, 16)).astype(np.float32)
    for pairs in (False, True):
        y = ref.rotate(x, cos, sin, pairs)
        for t in range(3):
            for p in range(16):
                a, b = (2 * p, 2 * p + 1) if pairs else (p, p + 16)
                w = (x[t, 1, a] + 1j * x[t, 1, b]) * complex(cos[t, p], sin[t, p])
                assert abs(y[t, 1, a] - w.real) <= abs(w) * 2.0 ** -8 and abs(y[t, 1, b] - w.imag) <= abs(w) * 2.0 ** -8
        assert np.array_equal(y[..., 32:], x[..., 32:])


def test_reference_attention():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 2, 8)), rng.standard_normal((9, 8)), rng.standard_normal((9, 8))
    out, reach, mass = ref.attention(q, k, v, [-1, 4, 8], 0.5, window=2, sinks=1, softcap=2.0)
    assert (out[0] == 0).all()
    for i, keys in ((1, [0, 3, 4]), (2, [0, 7, 8])):
        for r in range(2):
            w = [math.exp(2.0 * math.tanh(0.5 * float(q[i, r] @ k[j]) / 2.0)) for j in keys]
            want = sum(a * v[j] for a, j in zip(w, keys)) / sum(w)
            assert np.allclose(out[i, r], want, rtol=1e-12, atol=1e-12)
            assert mass[i, r] >= np.abs(want).max() and reach[i, r] >= max(abs(float(q[i, r] @ k[j])) for j in keys)
