"""The plans of packed and linear calls on the CPU (tests/c/pack_probe.cpp: the
host side over recording launchers): every token in one item, none of two long
sequences together, shares that make up whole tiles, nothing past the workspace."""
import ctypes
import functools
import os
import subprocess
import tempfile

import numpy as np
import pytest

import paper_2606_25041_amd as ws

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCES = [os.path.join(ROOT, "tests", "c", "pack_probe.cpp")] + [
    os.path.join(ROOT, "paper_2606_25041_amd", "csrc", f) for f in ("ws_api.cpp", "ws_api_pack.cpp", "ws_api_linear.cpp")]


@functools.lru_cache(maxsize=None)
def probe():
    with tempfile.TemporaryDirectory() as tmp:
        so = os.path.join(tmp, "pack_probe.so")
        subprocess.run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", *SOURCES, "-o", so], check=True)
        return ctypes.CDLL(so)


def ints(x):
    return None if x is None else np.ascontiguousarray(x, np.int32)


def ptr(x):
    return None if x is None else ctypes.c_void_p(x.ctypes.data)


def lengths(rng):
    """Lengths of some sequences, short and long, some empty."""
    top = int(np.exp(rng.uniform(np.log(2), np.log(30000))))
    n = int(np.exp(rng.uniform(0, np.log(rng.choice((4, 40, 900))))))
    lens = np.exp(rng.uniform(0, np.log(top), n)).astype(int)
    lens[rng.random(n) < 0.1] = 0
    return lens if lens.sum() else np.array([1])


def layout(rng, lens):
    """Sequence offsets; blocks and segment starts half of the time."""
    seqs = np.concatenate(([0], np.cumsum(lens)))
    if rng.random() < 0.5:
        return ints(seqs), None, None
    cuts = set(seqs.tolist()) | set(rng.integers(0, seqs[-1] + 1, rng.integers(0, 60)).tolist())
    blocks = np.array(sorted(cuts) if rng.random() < 0.5 else sorted(list(cuts) + [int(seqs[-1])]))   # (an empty block)
    text = None
    if rng.random() < 0.5:
        text = blocks[:-1] + (rng.random(len(blocks) - 1) * (np.diff(blocks) + 1)).astype(int)
    return ints(seqs), ints(blocks), ints(text)


def check_items(items, seqs, size):
    items = items[np.argsort(items[:, 0])]
    assert (items[:, 1] - items[:, 0] >= 1).all() and (items[:, 1] - items[:, 0] <= size).all()
    assert items[0, 0] == 0 and items[-1, 1] == seqs[-1] and (items[1:, 0] == items[:-1, 1]).all()
    lens = np.diff(seqs)
    for a, e in items:
        own = [s for s in range(len(lens)) if lens[s] and seqs[s] < e and seqs[s + 1] > a]
        # of several sequences only where each lies whole in it
        assert len(own) == 1 or all(a <= seqs[s] and seqs[s + 1] <= e for s in own), (a, e, own)


@pytest.mark.parametrize("seed", range(40))
def test_packed_plans(seed):
    rng = np.random.default_rng(seed)
    lens = lengths(rng)
    seqs, blocks, text = layout(rng, lens)
    n, total = len(lens), int(seqs[-1]) + int(rng.integers(0, 50))
    hq, hkv = [(8, 8), (32, 8), (64, 8), (8, 1), (5, 5), (40, 8)][seed % 6]
    probe().probe_cus(int(rng.choice((256, 256, 80))))
    nb = 0 if blocks is None else len(blocks) - 1
    out, items = (ctypes.c_int * 5)(), np.zeros((512, 2), np.int32)
    assert probe().probe_prefill(ptr(seqs), n, ptr(blocks), nb, ptr(text), total, hq, hkv, 128, out, ptr(items)) == 0
    kg, count, table, size, launched = out
    assert launched == 1 and size == (128 if kg == 2 else 256)
    if table:
        assert count == table
        check_items(items[:table], seqs, size)
    else:
        assert count == -(-int(seqs[-1]) // size)
    need = ws.library().ws_prefill_packed_bwd_workspace_bytes(total, hq, hkv)
    least = (8 * hq * total + 255) // 256 * 256 + 8 * total
    for size in (need, least):
        rows, keys = np.zeros((512, 2), np.int32), np.zeros((320, 2), np.int32)
        shares, sums, used = np.zeros((320, 3), np.int32), np.zeros((320, 3), np.int32), ctypes.c_int64()
        assert probe().probe_bwd(ptr(seqs), n, ptr(blocks), nb, ptr(text), total, hq, hkv, ctypes.c_int64(size), out, ptr(rows), ptr(keys),
                                 ptr(shares), ptr(sums), ctypes.byref(used)) == 0
        nrows, rtable, nkeys, ktable, nsums = out
        assert used.value <= size
        if rtable:
            check_items(rows[:nrows], seqs, 128)
        if not ktable:
            assert nkeys == -(-int(seqs[-1]) // 128) and nsums == 0
            continue
        tiles = {}
        for (a, e), (slot, part, parts) in zip(keys[:nkeys], shares[:nkeys]):
            tiles.setdefault((a, e), []).append((part, parts, slot))
        check_items(np.array(list(tiles)), seqs, 128)
        slots = []
        for tile, got in tiles.items():
            parts = got[0][1]
            assert sorted(p for p, _, _ in got) == list(range(parts)) and all(k == parts for _, k, _ in got)
            if parts > 1:
                first = min(s for _, _, s in got)
                assert sorted((s, p) for p, _, s in got) == [(first + i, i) for i in range(parts)]
                assert (tile[0], first, parts) in {tuple(x) for x in sums[:nsums]}
                slots += [s for _, _, s in got]
        assert len(set(slots)) == len(slots) and nsums == sum(g[0][1] > 1 for g in tiles.values())
        assert size == need or not slots


def test_long_axes_fall_back():
    probe().probe_cus(256)
    out, items = (ctypes.c_int * 5)(), np.zeros((512, 2), np.int32)
    for lens in ([300] * 400, [(1 << 24) + 5]):
        seqs = ints(np.concatenate(([0], np.cumsum(lens))))
        assert probe().probe_prefill(ptr(seqs), len(lens), None, 0, None, int(seqs[-1]), 8, 8, 128, out, ptr(items)) == 0
        assert out[2] == 0 and out[1] == -(-int(seqs[-1]) // 256)


@pytest.mark.parametrize("seed", range(40))
def test_linear_plans(seed):
    rng = np.random.default_rng(100 + seed)
    lens = lengths(rng)
    seqs = ints(np.concatenate(([0], np.cumsum(lens))))
    n, total = len(lens), int(seqs[-1]) + int(rng.integers(0, 50))
    hq, hkv = [(8, 8), (32, 8), (64, 8), (8, 1), (5, 5), (24, 24), (600, 600)][seed % 7]
    d = int(rng.choice((64, 128)))
    size = ws.library().ws_linear_workspace_bytes(n, total, hq, hkv, d)
    for back, state, flags in ((0, 0, 0), (0, 1, 0), (0, 1, 1), (0, 1, 2), (1, 0, 0), (1, 1, 0)):
        kinds, out, used = (ctypes.c_int * 9)(), (ctypes.c_int * 20)(), ctypes.c_int64()
        assert probe().probe_linear(ptr(seqs), n, total, hq, hkv, d, back, state, flags, kinds, out, ctypes.byref(used)) == 0
        assert used.value <= size
        order = list(kinds)[:list(kinds).index(0)]
        empty = (lens == 0).any()
        for i, kind in enumerate([2, 12] if back else [2]):
            cell, ncells, work, per_xcd, sets = out[5 * i:5 * i + 5]
            assert cell % 32 == 0 and ncells == -(-int(seqs[-1]) // cell) and ncells <= 1024
            assert per_xcd * 8 >= work and sets == hq // hkv
            crossing = any(a < e and a // cell != (e - 1) // cell for a, e in zip(seqs, seqs[1:]))
            at = order.index(kind)
            assert (at > 0 and order[at - 1] == kind - 1) == crossing
        if not back:
            reads, writes = state and flags != 1, state and flags != 2
            apart = out[2] > out[1] * hkv   # query heads with work-groups of their own
            assert out[2] == out[1] * (hq if apart else hkv) and (not apart or out[2] <= (512 if d == 128 else 1024))
            late = reads and writes and (1 in order or apart)
            assert (4 in order) == late and (3 in order) == (bool(empty) and writes and (late or not reads))
        else:
            assert (3 in order) == (bool(empty) and bool(state))
