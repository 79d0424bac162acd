"""Bounds on the scores that tpq_kv_attention refuses (before anything is enqueued, so that the made-up pointers are never followed):
cap tanh(s / cap) is off by 2^-22 of the bound, so that with a bound of 10^6 scores differ by 0.2 from what they are."""
import ctypes

import numpy as np
import pytest

import paper_2411_07942_amd as tpq


def _p(i):
    return ctypes.c_void_p(0x100000 * i)


def attention(cap, rows=0):
    L = tpq.kv_layout_init(2, 128, 64, 16)
    b = tpq._KvBatch(_p(10), _p(11), _p(12), 4, 8, 5, 100, rows, 64, 0)
    return tpq._load().tpq_kv_attention(ctypes.byref(L), _p(1), ctypes.byref(b), _p(2), 512, 4, 0.1, 0, 0, cap, _p(3), 512, _p(4), 1 << 40, None)


@pytest.mark.parametrize("cap", [1e-45, 1e-30, 2.0 ** -21, 1025.0, 1e4, 1e6, 1e30, 3e38, -1e-3])
def test_refused(cap):
    assert attention(cap) == attention(cap, 20) == tpq.ERR_SHAPE


@pytest.mark.parametrize("cap", [0.0, -0.0, 2.0 ** -20, 30.0, 50.0, 1024.0])
def test_taken(cap):
    assert attention(cap) == tpq.OK  # (no rows)


def test_error_of_a_bounded_score():
    """2^-22 of the bound (fp32 in this order: exp 2^-23, 1 + exp 2^-24, reciprocal 2^-23, product and sum 2^-24 each)."""
    for cap in (1.0, 50.0, 1024.0, 1e6):
        c, x = np.float32(cap), np.linspace(-3, 3, 20001).astype(np.float32)
        got = c - np.float32(2) * c * (np.float32(1) / (np.exp(np.float32(2) * x / c * np.float32(1)) + np.float32(1)))
        assert np.abs(got - cap * np.tanh(x.astype(np.float64) / cap)).max() <= cap * 2.0 ** -22
