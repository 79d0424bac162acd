"""The cache of keys and values in 4 bits and the attention over it: what is measured, and in plain form.

A case is one pass of one of two paths, at one size:

  append  new tokens' keys and values rotated by their positions, quantised and written to
          their pages, the queries rotated beside them; then the same tokens read back out of the
          cache (as a sequence is handed to another device)
  attend  attention of a batch's new tokens over the cache: one token per sequence (decode),
          a few (a draft's verification), a chunk or a whole prompt; a sliding window, first
          tokens that stay visible and a bound on the scores where the case has them

Quantiser, per token, head and group of G features: zero = minimum, scale = bf16((max - min) / 15),
code = rint((x - zero) * (1 / scale)) in 0..15, value = code * scale + zero, in fp32.

The cache is one buffer of pages; a page holds `page` tokens of every key/value head, a head's
cell being

  K codes  [page][D / 2] bytes   dword (g, kk) of a row, g < 4, kk < D / 32, at g * D / 32 + kk: features
                                 32 kk + 8 g + 0..7, feature 2 t in bits 4 t, feature 2 t + 1 in bits 16 + 4 t
  V codes  [page][D / 2] bytes   chunk m < 16 of D / 32 bytes: features 16 n + m, n < D / 16, in bits 4 n
  K meta   [D / G][page]         a group's scale and zero, bf16 each
  V meta   [D / G][page]

A sequence's tokens lie in the pages that its row of the table lists, token j at j % page of entry
j / page; of its len tokens the last n are the batch's new ones.

Sizes are those of the repository's workloads on one device of eight (Llama-2-13B: 5 heads of 128;
Gemma-2-27B: 4 query heads, 2 key/value heads, window 4096, scores bounded by 50) or on a whole
device, and generic ones.
"""
from __future__ import annotations

import math

import torch

own = False


def listed():
    return [
        # a decode step of 64 sequences, one device of eight (Gemma-2-27B): launch and latency
        dict(name="append_token", path="append", B=64, new=1, lo=512, hi=8192, Hq=4, Hkv=2, D=128, G=128, page=16,
             rot=128, pairs=False),
        # a 2048-token prompt, one device of eight (Llama-2-13B)
        dict(name="append_prompt", path="append", B=1, new=2048, lo=2048, hi=2048, Hq=5, Hkv=5, D=128, G=128, page=64,
             rot=128, pairs=False),
        # a serving step's mix of prompts and single tokens: ragged, small groups, a partial rotation of pairs
        dict(name="append_ragged", path="append", B=37, new=777, lo=800, hi=5000, Hq=32, Hkv=8, D=64, G=32, page=16,
             rot=32, pairs=True),
        # one user's token after a short text: latency alone
        dict(name="attend_one", path="attend", B=1, new=1, lo=641, hi=641, Hq=5, Hkv=5, D=128, G=128, page=16, window=0,
             sinks=0, cap=0.0),
        # a decode step of 64 sequences in a local layer, one device of eight (Gemma-2-27B)
        dict(name="attend_gemma", path="attend", B=64, new=1, lo=512, hi=8192, Hq=4, Hkv=2, D=128, G=128, page=16,
             window=4096, sinks=0, cap=50.0),
        # a decode step of 64 sequences, all 40 heads on one device: every head has keys of its own
        dict(name="attend_llama", path="attend", B=64, new=1, lo=1024, hi=4096, Hq=40, Hkv=40, D=128, G=128, page=64,
             window=0, sinks=0, cap=0.0),
        # a few very long contexts, grouped heads, smaller quantisation groups
        dict(name="attend_long", path="attend", B=3, new=1, lo=60001, hi=131072, Hq=32, Hkv=8, D=128, G=64, page=128,
             window=0, sinks=0, cap=0.0),
        # endless streams: a window of 1024 and 4 first tokens, the smallest groups
        dict(name="attend_sinks", path="attend", B=128, new=1, lo=20, hi=20000, Hq=32, Hkv=8, D=128, G=32, page=32,
             window=1024, sinks=4, cap=0.0),
        # a draft of 5 tokens verified for 16 sequences
        dict(name="attend_draft", path="attend", B=16, new=5, lo=300, hi=9000, Hq=32, Hkv=8, D=128, G=64, page=16,
             window=0, sinks=0, cap=0.0),
        # a 2048-token prompt, one device of eight (Llama-2-13B)
        dict(name="attend_prompt", path="attend", B=1, new=2048, lo=2048, hi=2048, Hq=5, Hkv=5, D=128, G=128, page=64,
             window=0, sinks=0, cap=0.0),
        # the last chunk of a long prompt on a whole device
        dict(name="attend_chunk", path="attend", B=1, new=4096, lo=16384, hi=16384, Hq=32, Hkv=8, D=128, G=128, page=64,
             window=0, sinks=0, cap=0.0),
        # a mixed batch, wide heads, window and sinks, odd lengths
        dict(name="attend_ragged", path="attend", B=9, new=600, lo=605, hi=5003, Hq=16, Hkv=2, D=256, G=128, page=16,
             window=701, sinks=3, cap=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    D = rng.choice([64, 128, 128, 128, 256])
    Hkv = rng.choice([1, 2, 4, 5, 8, 8, 40])
    R = rng.choice([1, 2, 3, 4, 8, 16]) if Hkv <= 8 else 1
    c = dict(B=1, new=1, lo=1, hi=1, Hq=R * Hkv, Hkv=Hkv, D=D, G=rng.choice([g for g in (32, 64, 128, 256) if g <= D]),
             page=rng.choice([16, 16, 32, 64, 128]))
    path = rng.choice(["append", "attend", "attend", "attend"])
    kind = rng.choice(["one", "one", "few", "many"])
    budget = 1 << rng.randint(12, 18)                       # tokens in the cache, all sequences
    if kind == "one":
        c["B"] = _log(rng, 1, 256)
    elif kind == "few":
        c["B"], c["new"] = _log(rng, 1, 64), rng.randint(2, 16)
    else:
        c["B"], c["new"] = _log(rng, 1, 16), _log(rng, 17, 2048)
        budget = min(budget, 1 << 15)
    c["hi"] = max(c["new"], min(budget // c["B"], 131072 if kind == "one" else 16384) // (1 + Hkv // 16)) + rng.randint(0, 63)
    if path == "attend":                                    # scores of a pass: no more than the largest listed case's
        while c["B"] * c["Hq"] * c["new"] * c["hi"] * D > 1 << 37 and c["new"] > 1:
            c["new"] = (c["new"] + 1) // 2
    c["lo"] = max(1, int(c["hi"] * rng.choice([1.0, 0.5, 0.1])))
    if path == "append":
        c["rot"], c["pairs"] = rng.choice([0, D // 2, D, D]), rng.random() < 0.5
    else:
        c["window"] = rng.choice([0, 0, rng.randint(1, 4096)])
        c["sinks"] = rng.randint(0, 64) if c["window"] else 0
        c["cap"] = rng.choice([0.0, 0.0, 30.0])
    return dict(path=path, **c)


# ---- lengths: by the case alone -------------------------------------------------------------

def _lengths(case):
    """Tokens of each sequence, and how many of them are new: spread between the case's ends by the golden ratio.
    With more than one new token every third sequence of a batch has the full number, the others fewer."""
    B, lo, hi, new = case["B"], case["lo"], case["hi"], case["new"]
    lens = [hi if b == 0 else lo + int((hi - lo) * ((b * 0.6180339887) % 1.0)) for b in range(B)]
    n = [new if b % 3 == 0 else 1 + int((new - 1) * ((b * 0.7548776662) % 1.0)) for b in range(B)]
    return lens, [min(a, b) for a, b in zip(n, lens)]


# ---- inputs ---------------------------------------------------------------------------------

def _gen(seed, *more):
    g = torch.Generator(device="cuda")
    s = seed
    for v in more:
        s = s * 1_000_003 + v
    g.manual_seed(s % (1 << 62))
    return g


def _pack(codes, key):
    """Codes [..., D] (uint8, 0..15) of a head's rows -> [..., D / 2] bytes in the cache's order."""
    D = codes.shape[-1]
    lead = codes.shape[:-1]
    if key:
        c = codes.view(*lead, D // 32, 4, 4, 2).transpose(-4, -3).transpose(-1, -2)      # g, kk, odd, t
        c = c.reshape(*lead, D // 2, 2)
    else:
        c = codes.view(*lead, D // 16, 16).transpose(-1, -2).reshape(*lead, D // 2, 2)   # m, n
    return c[..., 0] | (c[..., 1] << 4)


def _random_cells(case, n_pages, key, seed):
    """What a cache of rotated keys (features of different ranges) or values holds: codes, scale and zero as
    quantised activations have them, without going through activations."""
    Hkv, D, page, ng = case["Hkv"], case["D"], case["page"], case["D"] // case["G"]
    g = _gen(seed, 5 if key else 6)
    codes = torch.randint(0, 256, (n_pages, Hkv, page * D // 2), generator=g, device="cuda", dtype=torch.uint8)
    width = torch.rand((n_pages, Hkv, ng, page), generator=g, device="cuda") * 2.0 + (3.0 if key else 2.0)
    scale = (width / 15.0).to(torch.bfloat16)
    zero = (-width * (0.4 + 0.2 * torch.rand((n_pages, Hkv, ng, page), generator=g, device="cuda"))).to(torch.bfloat16)
    return codes, torch.stack((scale, zero), -1).view(torch.uint8).reshape(n_pages, Hkv, -1)


def prepare(case, seed):
    B, Hq, Hkv, D, page = case["B"], case["Hq"], case["Hkv"], case["D"], case["page"]
    lens, new = _lengths(case)
    width = max(-(-n // page) for n in lens)
    n_pages = sum(-(-n // page) for n in lens) + 7
    order = torch.randperm(n_pages, generator=_gen(seed, 1), device="cuda").tolist()
    table, at = [], 0
    for n in lens:
        used = -(-n // page)
        table.append(order[at:at + used] + [0] * (width - used))
        at += used
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    T = starts[-1]
    s = dict(case=case, n_pages=n_pages, T=T, table=torch.tensor(table, dtype=torch.int32, device="cuda"),
             lens=torch.tensor(lens, dtype=torch.int32, device="cuda"),
             starts=torch.tensor(starts, dtype=torch.int32, device="cuda") if case["new"] > 1 else None)
    g = _gen(seed, 2)
    if case["path"] == "append":
        # queries, keys and values side by side, as the projection in front leaves them
        s["cache"] = torch.zeros(n_pages * Hkv * page * (D + 8 * (D // case["G"])), dtype=torch.uint8, device="cuda")
        qkv = torch.randn((T, Hq + 2 * Hkv, D), generator=g, device="cuda")
        qkv[:, :, :: max(D // 8, 1)] *= 8.0
        s["qkv"] = qkv.to(torch.bfloat16)
        s["Q_out"] = torch.empty((T, Hq, D), dtype=torch.bfloat16, device="cuda")
        s["K_out"] = torch.empty((T, Hkv, D), dtype=torch.float32, device="cuda")
        s["V_out"] = torch.empty((T, Hkv, D), dtype=torch.float32, device="cuda")
        if case["rot"]:
            half = case["rot"] // 2
            rate = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
            angle = torch.arange(max(lens), dtype=torch.float64, device="cuda")[:, None] * rate
            s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        else:
            s["cos"] = s["sin"] = None
    else:
        k, km = _random_cells(case, n_pages, True, seed)
        v, vm = _random_cells(case, n_pages, False, seed)
        s["cache"] = torch.cat((k, v, km, vm), -1).reshape(-1)
        s["Q"] = (torch.randn((T, Hq, D), generator=g, device="cuda") * 1.5).to(torch.bfloat16)
        s["out"] = torch.empty((T, Hq, D), dtype=torch.bfloat16, device="cuda")
    if own:
        import paper_2411_07942_amd as tpq
        L = s["L"] = tpq.kv_layout_init(Hkv, D, case["G"], page)
        s["batch"] = tpq.KvBatch(s["table"], s["lens"], s["starts"], max_new=case["new"], max_len=max(lens))
        if case["path"] == "attend":
            s["workspace"] = tpq.kv_attention_workspace(L, s["batch"], Hq, "cuda")
    return s


# ---- the passes -----------------------------------------------------------------------------

def run(s):
    if own:
        return _run_own(s)
    return _append(s) if s["case"]["path"] == "append" else _attend(s)


def _run_own(s):
    import paper_2411_07942_amd as tpq
    c = s["case"]
    if c["path"] == "append":
        Hq, Hkv = c["Hq"], c["Hkv"]
        qkv = s["qkv"]
        tpq.kv_append(s["L"], s["cache"], s["batch"], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], s["cos"], s["sin"], c["pairs"],
                      qkv[:, :Hq], s["Q_out"])
        tpq.kv_read(s["L"], s["cache"], s["batch"], s["K_out"], s["V_out"])
        return s["Q_out"], s["K_out"], s["V_out"]
    tpq.kv_attention(s["L"], s["cache"], s["batch"], s["Q"], s["out"], c["D"] ** -0.5, s["workspace"], c["window"], c["sinks"],
                     c["cap"])
    return s["out"]


def _positions(s):
    """Of every new token its sequence and its position there."""
    T, B = s["T"], s["case"]["B"]
    row = torch.arange(T, device="cuda")
    if s["starts"] is None:
        return row, s["lens"].long() - 1
    starts = s["starts"].long()
    b = torch.searchsorted(starts[1:].contiguous(), row, right=True)
    return b, s["lens"].long()[b] - (starts[b + 1] - row)


def _rotate(x, cos, sin, pairs):
    """x fp32 [T, H, D]; the first 2 * cos.shape[-1] features of each head."""
    h = cos.shape[-1]
    c, n = cos[:, None], sin[:, None]
    a, b = (x[..., 0:2 * h:2], x[..., 1:2 * h:2]) if pairs else (x[..., :h], x[..., h:2 * h])
    y, z = a * c - b * n, b * c + a * n
    turned = torch.stack((y, z), -1).flatten(-2) if pairs else torch.cat((y, z), -1)
    return torch.cat((turned, x[..., 2 * h:]), -1).to(torch.bfloat16).float()


def _quantise(x, G):
    """x fp32 [T, H, D] of bf16 values -> codes uint8 [T, H, D], scale and zero bf16 [T, H, D / G]."""
    g = x.unflatten(-1, (-1, G))
    zero = g.amin(-1) + 0.0
    # (a divisor on the device: a number would become a product with its reciprocal)
    scale = ((g.amax(-1) - zero) / torch.full((), 15.0, device="cuda")).to(torch.bfloat16).float()
    scale = torch.where(scale < 1e-30, torch.zeros_like(scale), scale)
    inv = torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))
    codes = torch.round((g - zero[..., None]) * inv[..., None]).clamp(0, 15).to(torch.uint8).flatten(-2)
    return codes, scale.to(torch.bfloat16), zero.to(torch.bfloat16)


def _cells(s):
    """The cache as [pages, heads, bytes of a cell] and the offsets of a cell's four parts."""
    c = s["case"]
    rows, meta = c["page"] * c["D"] // 2, 4 * c["page"] * (c["D"] // c["G"])
    return s["cache"].view(s["n_pages"], c["Hkv"], -1), (0, rows, 2 * rows, 2 * rows + meta, 2 * rows + 2 * meta)


def _append(s):
    c = s["case"]
    Hq, Hkv, D, G, page = c["Hq"], c["Hkv"], c["D"], c["G"], c["page"]
    b, pos = _positions(s)
    x = s["qkv"].float()
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    if s["cos"] is not None:
        cos, sin = s["cos"][pos], s["sin"][pos]
        q, k = _rotate(q, cos, sin, c["pairs"]), _rotate(k, cos, sin, c["pairs"])
    cells, at = _cells(s)
    pages, slot = s["table"].long()[b, pos // page], pos % page
    head = torch.arange(Hkv, device="cuda")[None, :, None]
    p, t = pages[:, None, None], slot[:, None, None]
    byte, group = torch.arange(D // 2, device="cuda"), torch.arange(D // G, device="cuda")

    def store(y, key):
        codes, scale, zero = _quantise(y, G)
        cells[p, head, at[0 if key else 1] + t * (D // 2) + byte] = _pack(codes, key)
        meta = torch.stack((scale, zero), -1).view(torch.uint8).view(*scale.shape, 4)
        where = at[2 if key else 3] + 4 * (group * page + t)
        cells[p[..., None], head[..., None], where[..., None] + torch.arange(4, device="cuda")] = meta
        return codes.float().unflatten(-1, (-1, G)) * scale.float()[..., None] + zero.float()[..., None]

    K, V = store(k, True).flatten(-2), store(v, False).flatten(-2)
    return q.to(torch.bfloat16), K, V


def _unpack(part, key, D):
    """Bytes [..., D / 2] of a head's rows -> codes fp32 [..., D]."""
    lead = part.shape[:-1]
    c = torch.stack((part & 15, part >> 4), -1)
    if key:
        c = c.view(*lead, 4, D // 32, 2, 4).transpose(-1, -2).transpose(-4, -3)   # kk, g, t, odd
    else:
        c = c.view(*lead, 16, D // 16).transpose(-1, -2)                          # n, m
    return c.reshape(*lead, D).float()


def _gathered(s):
    """Keys and values of every sequence, fp32 [B, heads, tokens, D], from its pages."""
    c = s["case"]
    D, G, page, B, Hkv = c["D"], c["G"], c["page"], c["B"], c["Hkv"]
    cells, at = _cells(s)
    got = cells[s["table"].long()].transpose(1, 2)                                # [B, heads, pages, bytes]

    def values(i, key):
        codes = _unpack(got[..., at[i]:at[i + 1]].reshape(B, Hkv, -1, page, D // 2), key, D)
        meta = got[..., at[i + 2]:at[i + 3]].contiguous().view(torch.bfloat16).float().view(B, Hkv, -1, D // G, page, 2)
        meta = meta.transpose(3, 4)
        x = codes.unflatten(-1, (-1, G)) * meta[..., 0, None] + meta[..., 1, None]
        return x.reshape(B, Hkv, -1, D)

    return values(0, True), values(1, False)


def _attend(s):
    c = s["case"]
    D, Hq, Hkv, B, new = c["D"], c["Hq"], c["Hkv"], c["B"], c["new"]
    R = Hq // Hkv
    K, V = _gathered(s)
    b, pos = _positions(s)
    first = torch.arange(B, device="cuda") if s["starts"] is None else s["starts"].long()[:-1]
    nth = torch.arange(s["T"], device="cuda") - first[b]
    q = torch.zeros((B, new, Hq, D), dtype=torch.float32, device="cuda")
    q[b, nth] = s["Q"].float()
    at = torch.full((B, new), -1, dtype=torch.long, device="cuda")
    at[b, nth] = pos
    q = q.view(B, new, Hkv, R, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, R * new, D)
    x = torch.matmul(q, K.transpose(-1, -2).contiguous()).view(B, Hkv, R, new, -1) * (D ** -0.5)
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    j, i = torch.arange(K.shape[2], device="cuda"), at[:, :, None]
    seen = j <= i
    if c["window"]:
        seen = seen & ((j > i - c["window"]) | (j < c["sinks"]))
    x = torch.where(seen[:, None, None], x, -math.inf)
    p = torch.exp(x - x.amax(-1, keepdim=True).clamp(min=-1e30))
    o = torch.matmul(p.view(B, Hkv, R * new, -1), V).view(B, Hkv, R, new, D) / p.sum(-1, keepdim=True).clamp(min=1e-30)
    return o.permute(0, 3, 1, 2, 4).reshape(B, new, Hq, D)[b, nth].to(torch.bfloat16)


# ---- work and exact results -----------------------------------------------------------------

def work(case):
    lens, new = _lengths(case)
    Hq, Hkv, D, T = case["Hq"], case["Hkv"], case["D"], sum(new)
    cell = D + 8 * (D // case["G"])
    if case["path"] == "append":
        moved = 2 * (Hq + 2 * Hkv) * D + 2 * Hq * D + 8 * Hkv * D + 2 * cell * Hkv + 4 * case["rot"]
        return dict(bytes=T * moved, flops=T * D * (3 * Hq + 17 * Hkv))
    w, sinks = case["window"], case["sinks"]
    keys = pairs = 0
    for n, m in zip(lens, new):
        lo = max(0, n - m - w + 1) if w else 0
        keys += n - lo + min(sinks, lo)
        for pos in (range(n - m, n) if w else ()):
            low = max(0, pos - w + 1)
            pairs += pos + 1 - low + min(sinks, low)
        if not w:
            pairs += m * (n - m) + m * (m + 1) // 2
    return dict(bytes=keys * Hkv * cell + T * Hq * D * 4 + 4 * sum(-(-n // case["page"]) for n in lens),
                flops=4.0 * D * Hq * pairs)


def exact(case, seed):
    """The same outputs from the definitions in 64 bits: one sequence at a time, rows of the cache taken apart by
    shifting bits out of whole numbers.  Where the quantiser's and the rotation's definition rounds a step to 32 bits (codes
    of values halfway between two levels go by it), the 64-bit result of that step is rounded."""
    s = prepare(case, seed)
    lens, new = _lengths(case)
    Hq, Hkv, D, G, page = case["Hq"], case["Hkv"], case["D"], case["G"], case["page"]
    f = dict(dtype=torch.float64, device="cuda")
    bf = lambda t: t.to(torch.bfloat16).double()  # noqa: E731
    f32 = lambda t: t.float().double()  # noqa: E731
    if case["path"] == "append":
        pos = torch.cat([torch.arange(n - m, n, device="cuda") for n, m in zip(lens, new)])
        x = s["qkv"].double()
        if case["rot"]:
            h = case["rot"] // 2
            i = torch.arange(h, device="cuda")
            first, second = (2 * i, 2 * i + 1) if case["pairs"] else (i, i + h)
            c, n = s["cos"].double()[pos][:, None], s["sin"].double()[pos][:, None]
            y = x[:, :Hq + Hkv].clone()
            y[..., first] = bf(f32(x[:, :Hq + Hkv, first] * c) - f32(x[:, :Hq + Hkv, second] * n))
            y[..., second] = bf(f32(x[:, :Hq + Hkv, second] * c) + f32(x[:, :Hq + Hkv, first] * n))
            x = torch.cat((y, x[:, Hq + Hkv:]), 1)
        g = x[:, Hq:].reshape(-1, 2 * Hkv, D // G, G)
        zero = g.min(-1, keepdim=True).values
        scale = bf(f32(f32(g.max(-1, keepdim=True).values - zero) / 15))
        level = f32(f32(g - zero) * f32(1 / scale.clamp(min=1e-30))).round().clamp(0, 15)
        back = (torch.where(scale < 1e-30, torch.zeros((), **f), level * scale) + zero).reshape(-1, 2 * Hkv, D)
        return x[:, :Hq], back[:, :Hkv], back[:, Hkv:]
    if sum(m * n for n, m in zip(lens, new)) * Hq > 1 << 32:
        return None
    d = torch.arange(D, device="cuda")
    kword, kbit = (d // 8 % 4) * (D // 32) + d // 32, 4 * (d % 8 // 2) + 16 * (d % 2)
    vbyte, vbit = (d % 16) * (D // 32) + d // 32, 4 * (d // 16 % 2)
    cell = page * (D + 8 * (D // G))
    cache = s["cache"].view(-1, Hkv, cell)
    out, at = [], 0
    for b, (n, m) in enumerate(zip(lens, new)):
        pages = cache[s["table"][b, :-(-n // page)].long()]
        half = page * D // 2
        words = pages[..., :half].contiguous().view(torch.int32).view(-1, Hkv, page, D // 8)
        k = (words[..., kword] >> kbit & 15).double()
        v = (pages[..., half:2 * half].reshape(-1, Hkv, page, D // 2)[..., vbyte].int() >> vbit.int() & 15).double()
        meta = pages[..., 2 * half:].contiguous().view(torch.bfloat16).view(-1, Hkv, 2, D // G, page, 2).double()
        meta = meta.repeat_interleave(G, dim=3).permute(0, 1, 2, 4, 3, 5)                # [.., K or V, page, D, 2]
        k = (k * meta[:, :, 0, ..., 0] + meta[:, :, 0, ..., 1]).transpose(0, 1).reshape(Hkv, -1, D)[:, :n]
        v = (v * meta[:, :, 1, ..., 0] + meta[:, :, 1, ..., 1]).transpose(0, 1).reshape(Hkv, -1, D)[:, :n]
        q = s["Q"][at:at + m].double().view(m, Hkv, Hq // Hkv, D)
        j, i = torch.arange(n, device="cuda"), torch.arange(n - m, n, device="cuda")[:, None]
        hidden = (j > i) if not case["window"] else (j > i) | ((j <= i - case["window"]) & (j >= case["sinks"]))
        rows = []
        for h in range(Hkv):
            x = (q[:, h].reshape(-1, D) @ k[h].T).view(m, Hq // Hkv, n) / math.sqrt(D)
            if case["cap"]:
                x = case["cap"] * torch.tanh(x / case["cap"])
            x = torch.softmax(x.masked_fill(hidden[:, None], -math.inf), -1)
            rows.append((x.view(-1, n) @ v[h]).view(m, Hq // Hkv, D))
        out.append(torch.stack(rows, 1).reshape(m, Hq, D))
        at += m
    return torch.cat(out)
