"""Whole-sequence calls whose token positions would pass 32 bits are refused, on
the CPU (the host side over recording launchers, tests/c/session_plan_probe.cpp)."""
import ctypes

import numpy as np
import pytest

import paper_2606_25041_amd as ws
from tests import session_plan_probe as probe

OK, SHAPE = 0, 2


def _prefill(seq, window):
    lib, off, kg = probe._lib(), np.array([[0, seq]], np.int32), ctypes.c_int(0)
    lib.probe_cus(256)
    p = ctypes.c_void_p(off.ctypes.data)
    if window:
        return lib.reach_prefill_window(1, 1, 1, 64, seq, 1, p, None, 0, 100, 0, 0, ctypes.byref(kg))
    return lib.reach_prefill(1, 1, 1, 64, seq, 1, p, None)


@pytest.mark.parametrize("window", (False, True))
def test_prefill(window):
    """Query tiles and key tiles end at most 255 tokens behind the sequence."""
    last = 2 ** 31 - 1 - 256
    assert _prefill(last, window) == OK
    for seq in (last + 1, 2 ** 31 - 64, 2 ** 31 - 1):
        assert _prefill(seq, window) == SHAPE, seq


@pytest.mark.parametrize("window", (False, True))
def test_gradients(window):
    """A work-group's row data is 4 bytes a token, addressed in 32 bits."""
    lib = probe._lib()
    for seq, want in ((2 ** 30 - 1, OK), (2 ** 30, SHAPE), (2 ** 31 - 1, SHAPE)):
        off = np.array([[0, seq]], np.int32)
        assert lib.reach_bwd(1, 1, 1, 64, seq, 1, ctypes.c_void_p(off.ctypes.data), int(window), 100) == want, seq
    for name in ("ws_prefill_window_bwd_workspace_bytes", "ws_workspace_bytes"):
        getattr(lib, name).restype = ctypes.c_size_t

    def need(seq):
        if window:
            return lib.ws_prefill_window_bwd_workspace_bytes(1, 1, 1, seq, 0, 100)
        return lib.ws_workspace_bytes(3, 1, 1, 1, seq, seq)
    assert need(2 ** 30 - 1) >= 8 * (2 ** 30 - 1)
    assert need(2 ** 30) == need(2 ** 31 - 1) == 0


@pytest.mark.parametrize("window", (None, 2 ** 31 - 1))
def test_steps(window):
    """The key tile that holds the last token ends below 2^31 (pages may be
    shared, so memory is no limit: 2^25 table entries of one page)."""
    lib, new, fake = probe._lib(), 3, 0x10000
    lib.probe_cus(256)
    table = np.zeros((1, 2 ** 25), np.int32)
    kv = ws.PagedKVDesc(fake, fake, fake, table.ctypes.data, 1, 64, table.shape[1], 1, 64)
    t = ws.Tensor4(fake, ws.WS_DTYPE_BF16, new * 64, 64, 64)
    last = 2 ** 31 - 1 - 128
    for n, want in ((last - new, OK), (last - new + 1, SHAPE), (2 ** 31 - 1 - new, SHAPE), (2 ** 31 - 1, SHAPE)):
        lens = np.array([n], np.int32)
        head = (t, t, t, ctypes.byref(kv), ctypes.c_void_p(lens.ctypes.data), ctypes.c_void_p(fake))
        tail = (ctypes.c_float(0.1), 0, t, None, ctypes.c_void_p(fake), ctypes.c_size_t(1 << 40), None)
        if window is None:
            got = lib.ws_block_causal_attn_fwd(*head, 1, new, 1, *tail)
        else:
            got = lib.ws_block_causal_attn_fwd_window(*head, None, None, None, None, 1, new, 1, 0, window, *tail)
        assert got == want, n
