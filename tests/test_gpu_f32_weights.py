"""f32 outputs of windowed calls and of steps over a 4-bit cache hold all 24 bits
of the softmax weights, through every kernel and kind of plan: inputs on which
one weight's rounding shows whole (tests/f32_weights.py)."""
import numpy as np
import pytest
import torch

import paper_2606_25041_amd as ws
from tests import f32_weights as fw
from tests import gpu_support as gs
from tests import session_plan_cases as cases
from tests import window_ref
from tests.test_gpu_window import _layout

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _pair(x):
    h = torch.as_tensor(np.asarray(x), dtype=torch.int32).contiguous()
    return h, h.to(DEV)


def _step(hq, hkv, d, new, caches, lens, starts, window, sinks, make_cache):
    B = len(caches)
    q = fw.queries(B * new + hq, B, new, hq, d)
    pages = sum(-(-c // 64) for c in caches)
    table, at = torch.zeros(B, max(1, max(-(-c // 64) for c in caches)), dtype=torch.int32), 0
    for b, c in enumerate(caches):
        n = -(-c // 64)
        table[b, :n] = torch.arange(at, at + n)
        at += n
    cache = make_cache(max(1, pages), hkv, d, table)
    real = lens or [new] * B
    pairs = [[p for p in ([0, c - 2] if c >= 4 else [0]) if p + 1 < c + n] for c, n in zip(caches, real)]
    kn, vn = torch.zeros(B, new, hkv, d, dtype=torch.bfloat16), torch.zeros(B, new, hkv, d, dtype=torch.bfloat16)
    for b, c in enumerate(caches):
        k, v = fw.keys(c + real[b], pairs[b], hkv, d)
        kn[b, :real[b]], vn[b, :real[b]] = k[c:], v[c:]
        if c:
            one = type(cache)(*([cache.pool] if hasattr(cache, "pool") else [cache.k_pool, cache.v_pool]), table[b:b + 1])
            ws.kv_append(one, [0], k[None, :c].to(DEV), v[None, :c].to(DEV))
    kw = {} if window is None else dict(window=window, sinks=sinks)
    out = ws.block_causal_attn_fwd(q.to(DEV), kn.to(DEV), vn.to(DEV), cache, _pair(caches), scale=1.0,
                                   out_dtype=torch.float32, text_starts=None if starts is None else _pair(starts),
                                   new_lens=None if lens is None else _pair(lens), **kw).cpu()
    checked = 0
    for b, c in enumerate(caches):
        n = real[b]
        lo, hi = window_ref.step_ranges(c, n, None if starts is None else starts[b], 2 ** 31 if window is None else window)
        ref, rows = fw.want(q[b, :n], pairs[b], lo, hi, sinks)
        if rows.any():
            assert fw.worst(out[b, :n][rows], ref[rows]) <= 1, b
        checked += int(rows.sum())
    assert checked * hq >= 96   # (rows enough that weights in two parts would not pass: tests/test_f32_weights.py)


@pytest.mark.parametrize("d", cases.DIMS)
@pytest.mark.parametrize("case", range(len(cases.STEPS4)))
def test_4bit_step(case, d):
    cls, hq, hkv, new, caches, lens, starts = cases.STEPS4[case]
    gs.say(f"[gpu] f32 weights, 4-bit step, {cls}, d {d}")

    def make(pages, hkv, d, table):
        return ws.PagedCache4.allocate(pages, hkv, d, table, device=DEV)
    _step(hq, hkv, d, new, caches, lens, starts, None, 0, make)


@pytest.mark.parametrize("d", cases.DIMS)
@pytest.mark.parametrize("case", range(len(cases.STEPS_WINDOW)))
def test_windowed_step(case, d):
    cls, hq, hkv, new, caches, lens, starts, window, sinks = cases.STEPS_WINDOW[case]
    gs.say(f"[gpu] f32 weights, windowed step, {cls}, d {d}")

    def make(pages, hkv, d, table):
        return ws.PagedCache.allocate(pages, hkv, d, table, device=DEV, fill_bits=gs.NAN_BITS)
    _step(hq, hkv, d, new, caches, lens, starts, window, sinks, make)


@pytest.mark.parametrize("d", cases.DIMS)
@pytest.mark.parametrize("paged", (False, True))
@pytest.mark.parametrize("case", range(len(cases.PREFILLS)))
def test_windowed_prefill(case, paged, d):
    groups, B, hq, hkv, L, blocks, text, window, sinks = cases.PREFILLS[case]
    gs.say(f"[gpu] f32 weights, windowed prefill, {groups} key groups, paged {paged}, d {d}")
    lay = [_layout(50 + 100 * b, L, blocks, text) for b in range(B)]
    q, at = fw.queries(B * L + hq, B, L, hq, d), [0, L // 2]
    k, v = (x[None].repeat(B, 1, 1, 1).to(DEV) for x in fw.keys(L, at, hkv, d))
    off = _pair(np.concatenate([x[0] for x in lay]))
    kw = dict(scale=1.0, out_dtype=torch.float32, window=window, sinks=sinks,
              text_starts=_pair(np.concatenate([x[1] for x in lay])) if text else None)
    if paged:
        per = -(-L // 64)
        cache = ws.PagedCache.allocate(B * per, hkv, d, torch.arange(B * per).flip(0).reshape(B, per), device=DEV)
        ws.kv_append(cache, [0] * B, k, v)
        out = ws.block_causal_prefill(q.to(DEV), None, None, off, cache=cache, **kw)
    else:
        out = ws.block_causal_prefill(q.to(DEV), k, v, off, **kw)
    out = out.cpu()
    for b in range(B):
        lo, hi = window_ref.ranges(lay[b][0][0], lay[b][1][0] if text else None, window)
        ref, rows = fw.want(q[b], at, lo, hi, sinks)
        assert rows.sum() > L // 2
        assert fw.worst(out[b][rows], ref[rows]) <= 1, b
