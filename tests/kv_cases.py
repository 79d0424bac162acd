"""Attention over the 4-bit cache on the GPU against the 64-bit reference, each call held to the bound of the kernel that its
rows go to."""
import numpy as np
import torch

import kv_reference as ref
import paper_2411_07942_amd as tpq
import test_gpu_kv as kv


def few_rows(c, R, max_new):
    """Whether the products take the codes themselves (tpq_kv_attention: 64 rows, 32 of 4 groups, 8 of 8)."""
    ng = c.D // c.G
    return max_new * R <= (64 if ng <= 2 else 32 if ng == 4 else 8)


def attend(c, R, single=False, window=0, sinks=0, cap=0.0, scale=None, max_len=None, q_scale=1.0, stored=None):
    """The call with a workspace of NaN and rows that were something else before, against the reference.  stored: tokens of each
    sequence that the cache holds (fewer than its length: the others lie past the table)."""
    D, H, T = c.D, c.heads, c.rows
    scale = D ** -0.5 if scale is None else scale
    q = ref.bf16(c.rng.standard_normal((T, H * R, D)).astype(np.float32) * q_scale)
    out = torch.full((T, H * R, D), 7.0, dtype=torch.bfloat16, device="cuda")
    batch = c.batch(single, max_len=max_len)
    ws = tpq.kv_attention_workspace(c.L, batch, H * R, "cuda").fill_(kv.GARBAGE)
    tpq.kv_attention(c.L, kv.dev(c.bytes), batch, kv.bf16_tensor(q), out, scale, ws, window, sinks, cap)
    got = out.double().cpu().numpy().reshape(T, H, R, D)
    few = few_rows(c, R, batch.max_new)
    for b, (n, m) in enumerate(zip(c.lens, c.new)):
        if m == 0:
            continue
        held = n if stored is None else stored[b]
        rows = slice(int(c.starts[b]), int(c.starts[b]) + m)
        for h in range(H):
            k, v = c.k[b][:held, h].astype(np.float64), c.v[b][:held, h].astype(np.float64)
            want, reach, mass = ref.attention(q[rows, h * R:(h + 1) * R].astype(np.float64), k, v, np.arange(n - m, n), scale, window, sinks, cap)
            wide = np.abs(v).max() * 2.0 ** -20 if held else 0.0
            lim = kv.bound(want, reach, mass, wide, D, max(n, 1), scale, few)
            err = np.abs(got[rows, h] - want)
            assert (err <= lim).all(), (b, h, float((err - lim).max()), float((err / (lim + 1e-30)).max()))
    return got
