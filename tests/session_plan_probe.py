"""Which kernel and plan a windowed call or a step over a 4-bit cache reaches
(tests/c/session_plan_probe.cpp: the library's host side over recording
launchers), on the CPU, for a given number of compute units."""
import ctypes
import functools
import os
import subprocess
import tempfile
from types import SimpleNamespace

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCES = [os.path.join(ROOT, "tests", "c", "session_plan_probe.cpp")] + [
    os.path.join(ROOT, "paper_2606_25041_amd", "csrc", f) for f in ("ws_api.cpp", "ws_api4.cpp")]


@functools.lru_cache(maxsize=None)
def _lib():
    with tempfile.TemporaryDirectory() as tmp:
        so = os.path.join(tmp, "session_plan_probe.so")
        subprocess.run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", *SOURCES, "-o", so], check=True)
        return ctypes.CDLL(so)


def _ints(x):
    return None if x is None else np.ascontiguousarray(x, np.int32)


def _ptr(x):
    return None if x is None else ctypes.c_void_p(x.ctypes.data)


def _step(call, *args):
    out = (ctypes.c_int * 5)()
    assert call(*args, out) == 0
    return SimpleNamespace(kernel={1: "common", 2: "few rows"}[out[0]], f32=bool(out[1]), per_stream=bool(out[2]),
                           splits=out[3], merged=out[0] == 1 and bool(out[4]))


def step4(hq, hkv, d, new, caches, lens=None, f32=False, cus=256):
    """kernel, f32, per_stream (splits of its own for every stream), splits (of
    the stream that has most; few rows: its parts)."""
    _lib().probe_cus(cus)
    c, n = _ints(caches), _ints(lens)
    return _step(_lib().reach_step4, len(c), hq, hkv, d, new, _ptr(c), _ptr(n), int(f32))


def step_window(hq, hkv, d, new, caches, lens, window, sinks, f32=False, cus=256):
    _lib().probe_cus(cus)
    c, n = _ints(caches), _ints(lens)
    return _step(_lib().reach_step_window, len(c), hq, hkv, d, new, _ptr(c), _ptr(n), sinks, window, int(f32))


def prefill_window(hq, hkv, d, offsets, starts, window, sinks, paged=False, f32=False, cus=256):
    """Key groups of a work-group (1: 256-row tiles, 2: 128-row tiles).
    offsets [B][nb + 1], starts [B][nb] or None."""
    _lib().probe_cus(cus)
    off, text, kg = _ints(offsets), _ints(starts), ctypes.c_int(0)
    assert _lib().reach_prefill_window(off.shape[0], hq, hkv, d, int(off[0, -1]), off.shape[1] - 1, _ptr(off), _ptr(text),
                                       sinks, window, int(paged), int(f32), ctypes.byref(kg)) == 0
    return kg.value


def step_window_workspace(hq, hkv, d, new, caches, lens, window, sinks, f32=False, cus=256, given=-1):
    """Status, workspace bytes written and asked for, and the plan."""
    _lib().probe_cus(cus)
    c, n, out = _ints(caches), _ints(lens), (ctypes.c_int * 5)()
    used, need = ctypes.c_int64(0), ctypes.c_int64(0)
    rc = _lib().used_step_window(len(c), hq, hkv, d, new, _ptr(c), _ptr(n), sinks, window, int(f32), ctypes.c_int64(given),
                                 ctypes.byref(used), ctypes.byref(need), out)
    return rc, used.value, need.value, (bool(out[2]), out[3])


def step4_workspace(hq, hkv, d, new, caches, lens, f32=False, cus=256, given=-1):
    """The same of a step over a 4-bit cache (plan: few rows, per-stream splits)."""
    _lib().probe_cus(cus)
    c, n, out = _ints(caches), _ints(lens), (ctypes.c_int * 5)()
    used, need = ctypes.c_int64(0), ctypes.c_int64(0)
    rc = _lib().used_step4(len(c), hq, hkv, d, new, _ptr(c), _ptr(n), int(f32), ctypes.c_int64(given), ctypes.byref(used),
                           ctypes.byref(need), out)
    return rc, used.value, need.value, (out[0] == 2, bool(out[2]))
