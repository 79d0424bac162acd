"""KvBatch without a GPU: stand-ins for tensors on one, whose addresses nobody follows."""
import gc
import weakref

import pytest
import torch

import paper_2411_07942_amd as tpq


class OnGpu:
    dtype, is_cuda, device = torch.int32, True, torch.device("cuda", 0)

    def __init__(self, *shape):
        self.shape = torch.Size(shape)

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return id(self)


def test_a_batch_is_what_it_was_made_of():
    """Calls take the addresses that it was made with: another tensor in its place would not be read, and the first one's memory
    would be someone else's."""
    table, lens, starts = OnGpu(2, 3), OnGpu(2), OnGpu(3)
    batch = tpq.KvBatch(table, lens, starts, max_new=5, max_len=40)
    assert (batch.table, batch.lens, batch.starts, batch.max_new, batch.max_len) == (table, lens, starts, 5, 40)
    for name, value in (("table", OnGpu(2, 3)), ("lens", OnGpu(2)), ("starts", None), ("max_new", 6), ("max_len", None)):
        with pytest.raises(AttributeError):
            setattr(batch, name, value)
    alive = [weakref.ref(t) for t in (table, lens, starts)]
    del table, lens, starts
    gc.collect()
    assert all(r() is not None for r in alive)
    assert tpq.KvBatch(OnGpu(2, 3), OnGpu(2)).max_len is None


@pytest.mark.parametrize("max_new,max_len", [(0, None), (-1, None), (1 << 31, None), ((1 << 32) + 1, None), (1, 0), (1, -5), (1, 1 << 32), (1, (1 << 32) + 7)])
def test_numbers_that_no_call_takes(max_new, max_len):
    """(cut to 32 bits, 2^32 + 1 new tokens would have been 1, and the others left out)"""
    with pytest.raises(AssertionError):
        tpq.KvBatch(OnGpu(2, 3), OnGpu(2), OnGpu(3), max_new, max_len)


def test_check_of_another_device(monkeypatch):
    """As the other calls: the stream that is waited for is the current device's, and says nothing of another one's work."""
    L = tpq.kv_layout_init(1, 64, 64, 16)
    monkeypatch.setattr(tpq, "_load", lambda: pytest.fail("not refused"))
    batch = tpq.KvBatch(OnGpu(2, 3), OnGpu(2))
    with pytest.raises(AssertionError):
        tpq.kv_check(L, torch.zeros(4 * L.page_bytes, dtype=torch.uint8), batch, 2)      # not on a GPU
    cache = OnGpu(4 * L.page_bytes)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(AssertionError):
        tpq.kv_check(L, cache, batch, 2)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    cache.device = torch.device("cuda", 1)
    with pytest.raises(AssertionError):
        tpq.kv_check(L, cache, batch, 2)
