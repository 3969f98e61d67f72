"""Which page table entries an append to a bf16 cache needs, on the CPU: those of
the positions that it writes (device pointers are fake and never dereferenced; a
call that passes validation ends in the launch's error)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2606_25041_amd as ws

if torch.cuda.device_count() > 0:
    pytest.skip("uses fake device pointers; CPU-only module", allow_module_level=True)

FAKE = 0x10000
OK, SHAPE, PAGE, CAPACITY, HIP = 0, 2, 6, 7, 10


def append(table, lens, new, new_lens=None, pages=6):
    table, lens = np.ascontiguousarray(table, np.int32), np.asarray(lens, np.int32)
    t = ws.Tensor4(FAKE, ws.WS_DTYPE_BF16, new * 256, 256, 128)
    kv = ws.PagedKVDesc(FAKE, FAKE, FAKE, table.ctypes.data, pages, 64, table.shape[1], 2, 128)
    head = (ctypes.byref(kv), len(lens), lens.ctypes.data, FAKE)
    if new_lens is None:
        return ws.library().ws_kv_append(*head, new, t, t, None)
    nl = np.asarray(new_lens, np.int32)
    return ws.library().ws_kv_append_varlen(*head, nl.ctypes.data, FAKE, new, t, t, None)


@pytest.mark.parametrize("varlen", (False, True))
def test_pages_that_left_the_window_may_be_gone(varlen):
    """A session whose expired pages were given back commits its next block."""
    lens, new = [6400, 300], 70
    nl = [new, new] if varlen else None
    table = np.full((2, 102), -1)
    table[0, 100:102] = 4, 5          # positions 6400 .. 6469
    table[1, 4:6] = 2, 3              # 300 .. 369
    assert append(table, lens, new, nl) in (OK, HIP)
    for b, p in ((0, 100), (0, 101), (1, 4), (1, 5)):
        for bad in (-1, 6):
            broken = table.copy()
            broken[b, p] = bad
            assert append(broken, lens, new, nl) == PAGE, (b, p, bad)
    assert append(table[:, :101], lens, new, nl) == CAPACITY
    if varlen:   # a stream that commits nothing needs no page
        assert append(np.full((2, 102), -1), lens, new, [0, 0]) in (OK, HIP)
        assert append(table[:, :99], lens, new, [0, 0]) == CAPACITY


def test_positions_past_32_bits_are_refused():
    """The kernel counts positions in 32 bits (pages may be shared, so memory is
    no limit): 2^25 pages of one physical page."""
    table = np.zeros((1, 2 ** 25 + 1), np.int32)
    last = 2 ** 31 - 1
    assert append(table, [last - 5], 5) in (OK, HIP)
    assert append(table, [last - 5], 6) == SHAPE
    assert append(table, [last - 5], 6, [5]) in (OK, HIP)
    assert append(table, [last - 5], 6, [6]) == SHAPE
