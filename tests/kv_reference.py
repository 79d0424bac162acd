"""Plain implementations for the tests of the 4-bit cache of keys and values: rotation and quantiser in the 32-bit steps that
their definitions state, the cache's byte order, and attention in 64 bits.  numpy only, on the CPU; the quantiser is the oracle's."""
import numpy as np

import oracle
import workloads as wl


def bf16(x):
    """fp32 -> nearest bf16 value (ties to even), as fp32."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    u = (u + 0x7FFF + ((u >> 16) & 1)) >> 16
    return (u.astype(np.uint32) << 16).view(np.float32)


def bits(x):
    """fp32 array of bf16 values -> their patterns."""
    return (np.ascontiguousarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)


def rotate(x, cos, sin, pairs):
    """x fp32 [T, H, D] of bf16 values; cos, sin fp32 [T, rot / 2]: a rotation of rot features of every head."""
    h = cos.shape[-1]
    i = np.arange(h)
    first, second = (2 * i, 2 * i + 1) if pairs else (i, i + h)
    c, s = cos[:, None].astype(np.float32), sin[:, None].astype(np.float32)
    y = x.copy()
    y[..., first] = bf16(x[..., first] * c - x[..., second] * s)
    y[..., second] = bf16(x[..., second] * c + x[..., first] * s)
    return y


def quantise(x, G):
    """x fp32 [T, H, D] of bf16 values -> codes uint8 [T, H, D], scale and zero bf16 patterns [T, H, D / G]."""
    T, H, D = x.shape
    m = oracle.encode(bits(x).reshape(T, H * D), np.zeros(0, np.int32), G)
    codes = np.stack((m.codes & 15, m.codes >> 4), -1).reshape(T, H, D)
    return codes, m.scale.reshape(T, H, D // G), m.zero.reshape(T, H, D // G)


def values(codes, scale, zero):
    """fp32 code * scale + zero, both steps rounded."""
    G = codes.shape[-1] // scale.shape[-1]
    s, z = (np.repeat(wl.bits_to_f32(v), G, axis=-1) for v in (scale, zero))
    return (codes.astype(np.float32) * s).astype(np.float32) + z


def nibble_of(D, key):
    """Where in a row each feature's nibble lies."""
    d = np.arange(D)
    if not key:
        return (d % 16) * (D // 16) + d // 16
    g, kk, j = d // 8 % 4, d // 32, d % 8
    return 8 * (g * (D // 32) + kk) + np.where(j % 2 == 0, j // 2, 4 + j // 2)


def row_bytes(codes, key):
    """Rows of codes [..., D] -> [..., D / 2] bytes."""
    nibbles = np.zeros_like(codes)
    nibbles[..., nibble_of(codes.shape[-1], key)] = codes
    return nibbles[..., 0::2] | (nibbles[..., 1::2] << 4)


def store(cache, n_pages, D, G, page, pages, slots, key, codes, scale, zero):
    """Rows [T, H, ..] into the cache (uint8, flat), token t at (pages[t], slots[t])."""
    T, H, _ = codes.shape
    half, ng = page * D // 2, D // G
    cells = cache.reshape(n_pages, H, -1)
    p, h = np.asarray(pages)[:, None, None], np.arange(H)[None, :, None]
    first = (0 if key else half) + np.asarray(slots)[:, None, None] * (D // 2)
    cells[p, h, first + np.arange(D // 2)] = row_bytes(codes, key)
    meta = np.stack((scale, zero), -1).astype(np.uint16).view(np.uint8).reshape(T, H, ng, 4)
    where = 2 * half + (0 if key else 4 * ng * page) + 4 * (np.arange(ng)[None, None, :] * page + np.asarray(slots)[:, None, None])
    cells[p[..., None], h[..., None], where[..., None] + np.arange(4)] = meta


def visible(pos, n, window, sinks):
    j = np.arange(n)
    seen = j <= pos
    if window:
        seen &= (j > pos - window) | (j < sinks)
    return seen


def attention(q, k, v, pos, scale, window=0, sinks=0, softcap=0.0):
    """q fp64 [m, R, D], k, v fp64 [n, D] of one head, pos [m]: fp64 [m, R, D], and per row what bounds of its error
    go by: the largest sum |q_d k_d| of a visible key, and sum of weights * |v|'s largest."""
    m, R, D = q.shape
    out, reach, mass = np.zeros((m, R, D)), np.zeros((m, R)), np.zeros((m, R))
    for i in range(m):
        seen = np.flatnonzero(visible(pos[i], k.shape[0], window, sinks))
        if seen.size == 0:
            continue
        s = scale * (q[i] @ k[seen].T)
        if softcap > 0:
            s = softcap * np.tanh(s / softcap)
        w = np.exp(s - s.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        out[i] = w @ v[seen]
        reach[i] = (np.abs(q[i]) @ np.abs(k[seen]).T).max(-1)
        mass[i] = w @ np.abs(v[seen]).max(-1)
    return out, reach, mass
