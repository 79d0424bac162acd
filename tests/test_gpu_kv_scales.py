"""Attention over the 4-bit cache with scales below and at zero."""
import pytest
import torch

import paper_2411_07942_amd as tpq
import test_gpu_kv as kv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cap", [0.0, 5.0])
@pytest.mark.parametrize("lens,new,R,D,G", [([300, 40], [1, 1], 4, 128, 128), ([3000, 40], [2, 1], 4, 128, 32), ([150, 37], [1, 1], 3, 256, 64),
                                            ([300, 90], [100, 90], 1, 128, 64), ([200, 70], [90, 70], 1, 256, 128), ([300, 20], [70, 20], 2, 64, 32)])
def test_negative_and_zero_scales(lens, new, R, D, G, cap):
    """A negative scale is the positive one with negated queries, to the bit; with a scale of 0 every key seen weighs the same."""
    c = kv.Cache(lens, new, 2, D, G, 16, seed=sum(lens) + D).fill()
    cache, batch = kv.dev(c.bytes), c.batch(max(new) == 1)
    Q = torch.randn((c.rows, 2 * R, D), device="cuda").to(torch.bfloat16)
    ws = tpq.kv_attention_workspace(c.L, batch, 2 * R, "cuda")

    def run(q, scale):
        out = torch.full_like(q, 7.0)
        tpq.kv_attention(c.L, cache, batch, q, out, scale, ws.fill_(kv.GARBAGE), 0, 0, cap)
        return out
    assert torch.equal(run(Q, -0.1), run(-Q, 0.1))
    flat = run(Q, 0.0)
    for b, (n, m) in enumerate(zip(lens, new)):
        for i in range(m):
            mean = torch.from_numpy(c.v[b][:n - m + i + 1]).double().mean(0)
            got = flat[int(c.starts[b]) + i].double().cpu().view(2, R, D)
            # (half a bf16 step; values in fp16 2^-11 of the largest, sums of at most 3000 / 32 + 64 steps 143 / 15 of 2^-24)
            lim = mean.abs() * 2.0 ** -8 + float(abs(c.v[b]).max()) * (2.0 ** -11 + 160 * 10 * 2.0 ** -24)
            assert ((got - mean[:, None]).abs() <= lim[:, None]).all()
