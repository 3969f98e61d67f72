"""Windowed sessions that commit by a call of its own: solver steps over a unit,
then ws_kv_append(_varlen) into a table whose expired pages are gone."""
import numpy as np
import pytest
import torch

import paper_2606_25041_amd as ws
from tests import gpu_support as gs
from tests import window_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _randn(seed, *shape):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).to(torch.bfloat16)


def _pair(x):
    h = torch.as_tensor(np.asarray(x), dtype=torch.int32).contiguous()
    return h, h.to(DEV)


@pytest.mark.parametrize("varlen", (False, True))
def test_solver_steps_then_a_commit(varlen):
    gs.say(f"[gpu] windowed session, commits of its own, varlen={varlen}")
    Hq, Hkv, D, window, sinks, B, unit = 8, 2, 128, 200, 70, 2, 90
    sizes = [[90, 40], [17, 90], [90, 1], [64, 63], [90, 90], [5, 77], [90, 88]] if varlen else [[unit, unit]] * 7
    sizes = 2 * sizes   # (pages expire from 392 tokens on)
    total = [sum(s[b] for s in sizes) for b in range(B)]
    per = -(-(max(total) + unit) // 64)
    pages = B * (2 + -(-window // 64) + 1 + -(-unit // 64) + 1)
    pool = ws.PagedCache.allocate(pages, Hkv, D, torch.full((B, per), -1), device=DEV, fill_bits=gs.NAN_BITS)
    free, table = list(range(pages)), np.full((B, per), -1)
    kv = [(_randn(b, total[b], Hkv, D), _randn(10 + b, total[b], Hkv, D)) for b in range(B)]
    at = [0] * B
    for n, real in enumerate(sizes):
        for b in range(B):
            for p in range(per):
                if table[b, p] >= 0 and 64 * p >= sinks and 64 * (p + 1) <= at[b] - window:
                    pool.k_pool[table[b, p]], pool.v_pool[table[b, p]] = float("nan"), float("nan")
                    free.append(int(table[b, p]))
                    table[b, p] = -1
            for p in range(at[b] // 64, -(-(at[b] + real[b]) // 64)):
                if table[b, p] < 0:
                    table[b, p] = free.pop(0)
        cache = ws.PagedCache(pool.k_pool, pool.v_pool, torch.from_numpy(table.copy()))
        lens = dict(new_lens=_pair(real)) if varlen else {}
        for solver in range(2):
            q, kn, vn = (_randn(100 * n + 10 * solver + i, B, unit, h, D) for i, h in enumerate((Hq, Hkv, Hkv)))
            out = ws.block_causal_attn_fwd(q, kn, vn, cache, _pair(at), window=window, sinks=sinks, **lens)
            for b in range(B):
                m, c = real[b], at[b]
                lo, hi = ref.step_ranges(c, m, None, window)
                want = ref.attend(q[b, :m], torch.cat((kv[b][0][:c], kn[b, :m])), torch.cat((kv[b][1][:c], vn[b, :m])), lo, hi,
                                  sinks, D ** -0.5)
                ref.check(f"unit {n} stream {b}", out[b, :m], want["out"])
        clean = torch.full((2, B, unit, Hkv, D), float("nan"), dtype=torch.bfloat16, device=DEV)
        for b in range(B):
            clean[0, b, :real[b]], clean[1, b, :real[b]] = (x[at[b]:at[b] + real[b]] for x in kv[b])
        ws.kv_append(cache, _pair(at), clean[0], clean[1], **lens)
        at = [x + y for x, y in zip(at, real)]
        assert (table < 0).any()
    torch.cuda.synchronize()
    for b in range(B):
        assert (table[b, :at[b] // 64] < 0).sum() >= 3   # pages expired
