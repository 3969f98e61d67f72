"""Plans of windowed calls and of steps over a 4-bit cache, on the CPU: what a
launch writes stays inside the workspace it asked for, whatever the sizes and
the room, the parts cover the work, and only live pages have to exist."""
import ctypes
import functools
import os
import random
import subprocess
import tempfile

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCES = [os.path.join(ROOT, "tests", "c", "window_probe.cpp")] + [
    os.path.join(ROOT, "paper_2606_25041_amd", "csrc", f) for f in ("ws_api.cpp", "ws_api4.cpp")]
I64 = ctypes.c_int64


@functools.lru_cache(maxsize=None)
def _lib():
    with tempfile.TemporaryDirectory() as tmp:
        so = os.path.join(tmp, "window_probe.so")
        subprocess.run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", *SOURCES, "-o", so], check=True)
        lib = ctypes.CDLL(so)
    lib.ws_prefill_window_bwd_workspace_bytes.restype = ctypes.c_size_t
    lib.probe_cus(256)
    return lib


def _bwd(b, hq, hkv, d, seq, block, text, sinks, window, room):
    lib = _lib()
    need = lib.ws_prefill_window_bwd_workspace_bytes(b, hq, hkv, seq, sinks, window)
    least = -(-8 * b * hq * seq // 256) * 256 + 8 * b * seq
    given = {"full": need, "least": least, "half": max(least, (least + need) // 2), "more": 4 * need}[room]
    out, used = (ctypes.c_int * 3)(), I64(0)
    rc = lib.probe_bwd(b, hq, hkv, d, seq, block, text, sinks, window, I64(given), out, ctypes.byref(used))
    assert rc == 0
    return tuple(out), used.value, given, need


@pytest.mark.parametrize("room", ("full", "least", "half", "more"))
def test_gradient_parts_stay_in_the_workspace(room):
    g = random.Random(5)
    split = 0
    for _ in range(400):
        hkv, G = g.choice((1, 2, 3, 8)), g.choice((1, 3, 4, 8))
        seq = int(np.exp(g.uniform(0, np.log(70000))))
        args = (g.choice((1, 1, 2, 8)), hkv * G, hkv, g.choice((64, 128)), seq, g.choice((1, 174, 256, seq)),
                g.randint(0, 1), g.choice((0, 1, 64, 129, 700, 2 ** 31 - 1)),
                g.choice((0, 1, int(np.exp(g.uniform(0, 10))), 2 ** 31 - 1)), room)
        (sink_tiles, sink_parts, tile_parts), used, given, need = _bwd(*args)
        assert used <= given, args
        assert sink_parts >= 1 and tile_parts >= 1 and sink_tiles == min(-(-args[7] // 128), -(-seq // 128))
        split += sink_parts > 1 or tile_parts > 1
        if room == "least":
            assert (sink_parts, tile_parts) == (1, 1)
    assert room == "least" or split > 50


def test_sink_tiles_are_split_where_they_would_set_the_time():
    # 12 units of 174 tokens: 136 key tiles on 256 units, the sinks' seen by every row
    (_, sink_parts, _), _, _, _ = _bwd(1, 32, 8, 128, 2088, 174, 0, 5, 500, "full")
    assert sink_parts > 2
    # one sequence of one KV head: every tile in parts
    (_, sink_parts, tile_parts), _, _, _ = _bwd(1, 8, 1, 128, 3000, 174, 0, 5, 300, "full")
    assert sink_parts > tile_parts > 1


def _step_window(lens, table, pages, sinks, window, fuse, hq=8, hkv=2, d=128, new=3, room=-1):
    lib = _lib()
    lens = np.asarray(lens, np.int32)
    table = np.ascontiguousarray(table, np.int32)
    splits, need = ctypes.c_int(0), I64(0)
    rc = lib.probe_step_window(len(lens), hq, hkv, d, new, ctypes.c_void_p(lens.ctypes.data),
                               ctypes.c_void_p(table.ctypes.data), table.shape[1], pages, sinks, window, fuse, I64(room),
                               ctypes.byref(splits), ctypes.byref(need))
    return rc, splits.value, need.value


def test_a_windowed_step_needs_its_live_pages_only():
    OK, PAGE, CAPACITY, WORKSPACE = 0, 6, 7, 9
    n, sinks, window = 6400, 65, 200   # pages 0, 1 and those of 6200..6399; new tokens in page 100
    table = np.full((1, 101), -1)
    table[0, [0, 1]] = 0, 1
    table[0, 96:100] = 2, 3, 4, 5   # 6200 // 64 = 96
    assert _step_window([n], table, 6, sinks, window, 0)[0] == OK
    assert _step_window([n], table, 6, sinks, window, 1)[0] == PAGE   # a commit needs page 100
    table[0, 100] = 5
    assert _step_window([n], table, 6, sinks, window, 1)[0] == OK
    assert _step_window([n], table[:, :100], 6, sinks, window, 1)[0] == CAPACITY
    for page in (0, 1, 96, 97, 98, 99, 100):
        broken = table.copy()
        broken[0, page] = 6
        assert _step_window([n], broken, 6, sinks, window, 1)[0] == PAGE, page
    assert _step_window([n], np.full((1, 1), -1), 6, 0, 0, 0)[0] == OK   # nothing of the cache is seen
    rc, splits, need = _step_window([n], table, 6, sinks, 2 ** 31 - 1, 0)
    assert rc == PAGE
    full = np.zeros((1, 101))
    rc, splits, need = _step_window([n], full, 6, sinks, 2 ** 31 - 1, 0)
    assert rc == OK and splits > 1 and need > 0
    assert _step_window([n], full, 6, sinks, 2 ** 31 - 1, 0, room=need - 1)[0] == WORKSPACE
    # splits follow the live keys, not the history
    assert _step_window([n], full, 6, 0, 64, 0)[1] == 1


def _step4(lens, hq, hkv, d, new, room=-1):
    lib = _lib()
    lens = np.asarray(lens, np.int32)
    kind, per, nwg = ctypes.c_int(0), ctypes.c_int(0), ctypes.c_int(0)
    start, used, need = np.zeros(len(lens) + 1, np.int32), I64(0), I64(0)
    rc = lib.probe_step4(len(lens), hq, hkv, d, new, ctypes.c_void_p(lens.ctypes.data), I64(room), ctypes.byref(kind),
                         ctypes.byref(per), ctypes.byref(nwg), ctypes.c_void_p(start.ctypes.data), ctypes.byref(used),
                         ctypes.byref(need))
    return rc, kind.value, per.value, nwg.value, start, used.value, need.value


def test_4bit_steps_stay_in_the_workspace():
    g = random.Random(9)
    seen = set()
    for cus in (256, 304, 32, 1):
        _lib().probe_cus(cus)
        for _ in range(300):
            hkv, G, new = g.choice((1, 2, 3, 8, 24, 64, 300)), g.choice((1, 3, 4, 8, 16)), g.choice((1, 1, 2, 3, 17, 128, 512))
            b = g.choice((1, 1, 2, 4, 31, 32, 33))
            lens = [g.choice((0, 1, 63, 64, 65, int(np.exp(g.uniform(0, 12))))) for _ in range(b)]
            d = g.choice((64, 128))
            rc, kind, per, nwg, start, used, need = _step4(lens, hkv * G, hkv, d, new)
            assert rc == 0 and used <= need, (cus, lens, hkv, G, new, d)
            seen.add((kind, G * new <= 128))
            if b > 32 or G * new > 512:
                assert kind == 1
            if kind == 2:   # the line holds every stream's pages and new block, the work-groups all of it
                assert start[0] == 0 and (np.diff(start) == [-(-n // 64) + -(-new // 32) for n in lens]).all()
                assert (nwg - 1) * per < start[b] <= nwg * per and per >= 8
                nrb = -(-G * new // 32)
                assert nwg * hkv * nrb <= max(cus, hkv * nrb)
            if need:
                assert _step4(lens, hkv * G, hkv, d, new, need - 1)[0] == 9
    _lib().probe_cus(256)
    assert seen == {(1, False), (1, True), (2, False), (2, True)}


def test_positions_and_heads_past_32_bits_are_refused():
    OK, SHAPE, limit = 0, 2, 2 ** 31 - 1 - 128
    table = np.full((1, 1), -1)   # nothing of the cache is seen
    for n, want in ((limit - 3, OK), (limit - 2, SHAPE), (2 ** 31 - 1, SHAPE)):
        assert _step_window([n], table, 6, 0, 0, 0)[::2] == (want, 0), n
    # (heads x row blocks past 2^32: the share of a head was a division by zero)
    lib = _lib()
    lib.ws_step_workspace_bytes_4bit.restype = ctypes.c_size_t
    lens = np.array([100], np.int32)
    assert lib.ws_step_workspace_bytes_4bit(1, 1 << 30, 1 << 30, 128, ctypes.c_void_p(lens.ctypes.data), None) == 0
