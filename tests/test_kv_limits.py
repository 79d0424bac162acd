"""Calls of the 4-bit cache whose launch would not fit 2^32 threads are refused before anything is enqueued (so that the made-up
pointers are never followed)."""
import ctypes

import pytest

import paper_2411_07942_amd as tpq


def _p(i):
    return ctypes.c_void_p(0x100000 * i)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("rows", [0x7FFFFFFF, 1 << 30])
def test_more_rows_than_a_launch_takes(D, rows):
    lib = tpq._load()
    L = tpq.kv_layout_init(256, D, 64, 16)
    batch = tpq._KvBatch(_p(10), _p(11), _p(12), 4, 8, 1 << 20, 100, rows, 64, 0)
    E = 256 * D
    assert lib.tpq_kv_append(ctypes.byref(L), _p(1), ctypes.byref(batch), _p(2), E, _p(3), E, None, None, 0, 0, 0,
                             None, 0, 0, None, 0, None) == tpq.ERR_SHAPE
    assert lib.tpq_kv_read(ctypes.byref(L), _p(1), ctypes.byref(batch), 1, _p(2), E, _p(3), E, None) == tpq.ERR_SHAPE
