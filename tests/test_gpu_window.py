"""Attention through a sliding window with sinks: streaming steps, prefills and
gradients against float64 from the definition, every element within the bound
of the kernels' roundings (tests/window_ref.py).  Keys that no row sees hold
NaN, and the pages between the sinks and the window are gone from the table."""
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


def live_cache(seed, hkv, d, caches, extra, window, sinks):
    """A cache whose streams hold only what a windowed step may read (and room
    for `extra` new tokens): expired pages are -1 in the table, every slot that
    no row sees is NaN.  Returns it and the logical keys and values (NaN where
    not live) [n][hkv][d] of each stream."""
    per = max(-(-(c + extra) // 64) for c in caches)
    table = torch.full((len(caches), per), -1, dtype=torch.int32)
    kv = []
    for b, c in enumerate(caches):
        k, v = _randn(seed + 2 * b, c, hkv, d), _randn(seed + 2 * b + 1, c, hkv, d)
        p = torch.arange(c, device=DEV)
        hidden = (p >= sinks) & (p < c - window)
        k[hidden], v[hidden] = float("nan"), float("nan")
        kv.append((k, v))
        live = torch.zeros(per, dtype=torch.bool)
        for x in p[~hidden].tolist() + list(range(c, c + extra)):
            live[x // 64] = True
        table[b, live] = torch.arange(int(live.sum()), dtype=torch.int32) + int((table >= 0).sum())
    pages = int((table >= 0).sum()) + 1
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.where(table >= 0, order[table.clamp(min=0).long()], -1)
    cache = ws.PagedCache.allocate(pages, hkv, d, table, device=DEV, fill_bits=0x7FC1)
    for b, (k, v) in enumerate(kv):
        for page in range(per):
            n = min(64, k.shape[0] - 64 * page)
            if n > 0 and table[b, page] >= 0:
                cache.k_pool[table[b, page], :, :n] = k[64 * page:64 * page + n].transpose(0, 1)
                cache.v_pool[table[b, page], :, :n] = v[64 * page:64 * page + n].transpose(0, 1)
    return cache, kv


STEPS = [
    # Hq, Hkv, D, Lq, caches, new_lens, starts, window, sinks, f32
    (8, 2, 128, 1, [700, 0, 64, 129], None, None, 128, 4, False),
    (8, 2, 128, 1, [700, 0, 64, 129], None, [0, 0, 1, 0], 127, 64, True),
    (4, 4, 64, 1, [1000], None, [0], 0, 0, False),          # only itself
    (4, 4, 64, 33, [1000, 31], None, None, 0, 65, False),   # sinks and the block
    (16, 2, 64, 37, [5003, 1200, 64, 333, 0], None, None, 65, 1, True),
    (6, 2, 128, 100, [2500, 90], None, [60, 100], 63, 130, False),
    (6, 2, 128, 300, [640, 7], None, [0, 0], 100, 3, False),   # windows that leave the cache
    (64, 8, 128, 24, [9000, 4100, 3000, 17], [24, 1, 7, 20], [20, 0, 7, 3], 1000, 64, False),
    (64, 8, 128, 24, [9000, 4100, 3000, 17], [24, 1, 7, 20], None, 2048, 100, True),
    (24, 24, 128, 256, [2257], None, None, 1001, 4, False),
    (3, 1, 128, 90, [4000, 300], None, [10, 80], 2 ** 31 - 1, 5, False),    # everything
    (3, 1, 128, 90, [4000, 300], None, None, 50, 2 ** 31 - 1, True),        # all sinks
    (8, 1, 128, 5, [20000] * 3 + [40, 1] * 16, None, [0] * 35, 300, 65, False),   # lengths from memory
    (8, 8, 64, 520, [130], None, [500], 64, 64, False),
    # streams whose live keys differ much
    (16, 2, 128, 40, [9000, 17, 40, 0, 5], None, None, 4000, 64, False),
    (24, 24, 128, 200, [4000, 300, 30], [200, 33, 64], None, 2 ** 20, 3, True),
    (12, 4, 64, 90, [20000, 300, 300, 8], [90, 33, 64, 1], [80, 33, 0, 0], 9000, 100, False),
    (64, 8, 128, 243, [7000, 3011, 1400, 190], [145, 110, 163, 243], [140, 110, 160, 240], 3500, 65, False),
]


@pytest.mark.parametrize("case", range(len(STEPS)))
def test_step(case):
    Hq, Hkv, D, Lq, caches, lens, starts, window, sinks, f32 = STEPS[case]
    gs.say(f"[gpu] window step {case}: {STEPS[case]}")
    B = len(caches)
    cache, kv = live_cache(100 * case, Hkv, D, caches, Lq, window, sinks)
    q = _randn(7 + case, B, Lq, Hq, D)
    kn, vn = _randn(8 + case, B, Lq, Hkv, D), _randn(9 + case, B, Lq, Hkv, D)
    real = lens or [Lq] * B
    for b in range(B):
        kn[b, real[b]:], vn[b, real[b]:] = float("nan"), float("nan")
    kw = dict(out_dtype=torch.float32 if f32 else torch.bfloat16, want_lse=True, window=window, sinks=sinks,
              text_starts=None if starts is None else _pair(starts), new_lens=None if lens is None else _pair(lens))
    out, lse = ws.block_causal_attn_fwd(q, kn, vn, cache, _pair(caches), **kw)
    again, lse2 = ws.block_causal_attn_fwd(q, kn, vn, cache, _pair(caches), fuse_append=True, **kw)
    torch.cuda.synchronize()
    for b in range(B):
        n, c = real[b], caches[b]
        lo, hi = ref.step_ranges(c, n, None if starts is None else starts[b], window)
        k, v = torch.cat((kv[b][0], kn[b, :n])), torch.cat((kv[b][1], vn[b, :n]))
        want = ref.attend(q[b, :n], k, v, lo, hi, sinks, D ** -0.5, f32=f32)
        ref.check(f"out {b}", out[b, :n], want["out"])
        ref.check(f"lse {b}", lse[b, :, :n], want["lse"])
        assert torch.equal(out[b, :n], again[b, :n]) and torch.equal(lse[b, :, :n], lse2[b, :, :n]), b
        p = torch.arange(c, c + n, device=DEV)
        page = cache.page_table[b].long()[p // 64]
        assert torch.equal(cache.k_pool[page, :, p % 64], kn[b, :n])
        assert torch.equal(cache.v_pool[page, :, p % 64], vn[b, :n])
    written = int((~cache.k_pool[:, 0, :, 0].isnan()).sum())
    live = sum(int((~k[:, 0, 0].isnan()).sum()) for k, _ in kv)
    assert written == live + sum(real)   # nothing but the new tokens was written


@pytest.mark.parametrize("exponents", ((100,), (-100,), (96, 0), (30, -30, 0), (0, 0, 0, -60)))
@pytest.mark.parametrize("f32", (False, True))
def test_values_of_any_magnitude(exponents, f32):
    """Head dims whose values differ by up to 2^96, through split partials.  (The
    sums are unnormalised f32: 2^8 a weight x 3000 keys x 2^102 stay below 2^128.)"""
    gs.say(f"[gpu] window step, values of 2^{exponents} f32={f32}")
    D, window, sinks, caches, Lq = 128, 3000, 64, [9000, 3500], 9
    cache, kv = live_cache(5, 2, D, caches, Lq, window, sinks)
    unit = torch.exp2(torch.tensor([exponents[i % len(exponents)] for i in range(D)], device=DEV, dtype=torch.float64))
    unit = unit.to(torch.bfloat16)
    q, kn, vn = _randn(1, 2, Lq, 8, D), _randn(2, 2, Lq, 2, D), _randn(3, 2, Lq, 2, D) * unit
    cache.v_pool *= unit
    out, lse = ws.block_causal_attn_fwd(q, kn, vn, cache, _pair(caches), window=window, sinks=sinks, want_lse=True,
                                        out_dtype=torch.float32 if f32 else torch.bfloat16)
    torch.cuda.synchronize()
    for b, c in enumerate(caches):
        lo, hi = ref.step_ranges(c, Lq, None, window)
        want = ref.attend(q[b], torch.cat((kv[b][0], kn[b])), torch.cat((kv[b][1] * unit, vn[b])), lo, hi, sinks,
                          D ** -0.5, f32=f32)
        ref.check(f"out {b}", out[b], want["out"])
        ref.check(f"lse {b}", lse[b], want["lse"])


def _layout(seed, L, nblocks, text):
    """Block offsets [1][nb + 1] with empty blocks, and segment starts."""
    g = np.random.default_rng(seed)
    off = np.sort(np.concatenate(([0, L], g.integers(0, L + 1, nblocks - 1))))[None]
    starts = None
    if text:
        starts = np.array([[g.integers(s, e + 1) for s, e in zip(off[0, :-1], off[0, 1:])]])
    return off.astype(np.int32), None if starts is None else starts.astype(np.int32)


PREFILLS = [
    # B, Hq, Hkv, D, L, blocks, text, window, sinks, paged, f32
    (1, 2, 1, 64, 1, 1, False, 0, 0, False, True),
    (2, 4, 2, 128, 100, 7, True, 10, 3, False, False),
    (1, 4, 2, 64, 777, 20, False, 64, 64, True, False),
    (1, 3, 3, 128, 1300, 30, True, 100, 17, True, True),
    (2, 6, 2, 128, 1300, 150, True, 1, 0, False, False),     # more than 64 blocks a tile
    (1, 8, 2, 128, 2500, 9, False, 513, 130, False, False),
    (1, 40, 8, 128, 2600, 16, True, 777, 17, True, False),
    (1, 2, 2, 64, 3000, 3000, False, 255, 1, False, True),   # unit blocks: causal
    (1, 2, 2, 64, 3000, 1, True, 300, 200, False, False),    # one block with a segment
    (3, 2, 1, 128, 600, 5, True, 2 ** 31 - 1, 0, True, False),
    (1, 2, 1, 128, 900, 5, True, 7, 2 ** 31 - 1, False, True),
]


@pytest.mark.parametrize("case", range(len(PREFILLS)))
def test_prefill(case):
    B, Hq, Hkv, D, L, blocks, text, window, sinks, paged, f32 = PREFILLS[case]
    gs.say(f"[gpu] window prefill {case}: {PREFILLS[case]}")
    lay = [_layout(50 + case + 100 * b, L, blocks, text) for b in range(B)]
    off = _pair(np.concatenate([x[0] for x in lay]))
    starts = _pair(np.concatenate([x[1] for x in lay])) if text else None
    q, k, v = _randn(1 + case, B, L, Hq, D), _randn(2 + case, B, L, Hkv, D), _randn(3 + case, B, L, Hkv, D)
    kw = dict(out_dtype=torch.float32 if f32 else torch.bfloat16, want_lse=True, text_starts=starts, window=window,
              sinks=sinks)
    if paged:
        per = -(-L // 64)
        table = torch.randperm(B * per, generator=torch.Generator().manual_seed(case)).reshape(B, per)
        cache = ws.PagedCache.allocate(B * per, Hkv, D, table, device=DEV, fill_bits=0x7FC1)
        ws.kv_append(cache, [0] * B, k, v)
        out, lse = ws.block_causal_prefill(q, None, None, off, cache=cache, **kw)
    else:
        out, lse = ws.block_causal_prefill(q, k, v, off, **kw)
    torch.cuda.synchronize()
    for b in range(B):
        lo, hi = ref.ranges(lay[b][0][0], lay[b][1][0] if text else None, window)
        want = ref.attend(q[b], k[b], v[b], lo, hi, sinks, D ** -0.5, f32=f32)
        ref.check(f"out {b}", out[b], want["out"])
        ref.check(f"lse {b}", lse[b], want["lse"])


GRADS = [
    # B, Hq, Hkv, D, L, blocks, text, window, sinks, bf16
    (1, 2, 1, 64, 1, 1, False, 0, 0, False),
    (2, 4, 2, 128, 100, 7, True, 10, 3, True),
    (1, 4, 2, 64, 777, 20, False, 64, 64, False),
    (2, 6, 2, 128, 1300, 150, True, 1, 0, True),
    (1, 8, 2, 128, 2500, 9, False, 513, 130, True),
    (1, 8, 1, 128, 3000, 16, True, 300, 5, True),         # the sinks' tile in parts
    (1, 4, 1, 64, 3500, 3500, False, 255, 300, False),    # unit blocks, three sink tiles
    (8, 2, 1, 128, 900, 6, True, 200, 1, True),           # groups a multiple of the XCDs
    (1, 2, 2, 64, 1500, 1, True, 300, 200, True),
    (1, 3, 1, 128, 600, 5, True, 2 ** 31 - 1, 0, False),
    (1, 2, 1, 128, 900, 5, True, 7, 2 ** 31 - 1, True),
]


@pytest.mark.parametrize("case", range(len(GRADS)))
@pytest.mark.parametrize("room", ("full", "least"))
def test_gradients(case, room):
    B, Hq, Hkv, D, L, blocks, text, window, sinks, bf16 = GRADS[case]
    gs.say(f"[gpu] window gradients {case} {room}: {GRADS[case]}")
    lay = [_layout(70 + case + 100 * b, L, blocks, text) for b in range(B)]
    off = _pair(np.concatenate([x[0] for x in lay]))
    starts = _pair(np.concatenate([x[1] for x in lay])) if text else None
    q, k, v = _randn(1 + case, B, L, Hq, D), _randn(2 + case, B, L, Hkv, D), _randn(3 + case, B, L, Hkv, D)
    do = _randn(4 + case, B, L, Hq, D)
    win = dict(text_starts=starts, window=window, sinks=sinks)
    out, lse = ws.block_causal_prefill(q, k, v, off, want_lse=True, **win)
    need = -(-8 * B * Hq * L // 256) * 256 + 8 * B * L   # enough to run, unsplit
    workspace = torch.empty(need, dtype=torch.uint8, device=DEV) if room == "least" else None
    got = ws.block_causal_prefill_bwd(q, k, v, out, do, lse, off, workspace=workspace,
                                      grad_dtype=torch.bfloat16 if bf16 else torch.float32, **win)
    again = ws.block_causal_prefill_bwd(q, k, v, out, do, lse, off, workspace=workspace,
                                        grad_dtype=torch.bfloat16 if bf16 else torch.float32, **win)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, again))   # deterministic
    for b in range(B):
        lo, hi = ref.ranges(lay[b][0][0], lay[b][1][0] if text else None, window)
        want = ref.attend(q[b], k[b], v[b], lo, hi, sinks, D ** -0.5, dout=do[b])
        for name, x in zip(("dq", "dk", "dv"), got):
            assert x.dtype == (torch.bfloat16 if bf16 else torch.float32)
            ref.check(f"{name} {b}", x[b], want[name], bf16=bf16)


def test_a_billion_tokens_behind_the_window():
    """A session of 2^30 + 77 tokens of which the sinks and the window are left,
    in the last pages of a pool past 4 GiB."""
    gs.say("[gpu] window step at position 2^30")
    n, window, sinks, Hq, Hkv, D, Lq, pages = 2 ** 30 + 77, 1000, 70, 8, 8, 128, 5, 40000
    live = [(0, min(sinks, 64)), (64, sinks)] + [(p, min(p + 64, n)) for p in range((n - window) // 64 * 64, n, 64)]
    table = torch.full((1, (n + Lq + 63) // 64), -1, dtype=torch.int32)
    k_pool = torch.empty(pages, Hkv, 64, D, dtype=torch.bfloat16, device=DEV)
    v_pool = torch.empty_like(k_pool)
    ks, vs, at = [], [], []
    for i, (s, e) in enumerate(live):
        page = pages - 1 - i
        table[0, s // 64] = page
        k_pool[page], v_pool[page] = float("nan"), float("nan")
        lo = max(s, 0 if s < sinks else n - window)
        k, v = _randn(2 * i, e - lo, Hkv, D), _randn(2 * i + 1, e - lo, Hkv, D)
        k_pool[page, :, lo - s:e - s], v_pool[page, :, lo - s:e - s] = k.transpose(0, 1), v.transpose(0, 1)
        ks.append(k), vs.append(v), at.extend(range(lo, e))
    q, kn, vn = _randn(91, 1, Lq, Hq, D), _randn(92, 1, Lq, Hkv, D), _randn(93, 1, Lq, Hkv, D)
    cache = ws.PagedCache(k_pool, v_pool, table)
    out, lse = ws.block_causal_attn_fwd(q, kn, vn, cache, _pair([n]), text_starts=_pair([2]), window=window, sinks=sinks,
                                        want_lse=True)
    torch.cuda.synchronize()
    # the same with the gap left out: positions behind it move down
    lo, hi = ref.step_ranges(n, Lq, 2, window)
    gap = n - window - sinks
    assert at == list(range(sinks)) + list(range(n - window, n))
    want = ref.attend(q[0], torch.cat(ks + [kn[0]]), torch.cat(vs + [vn[0]]), lo - gap, hi - gap, sinks, D ** -0.5)
    ref.check("out", out[0], want["out"])
    ref.check("lse", lse[0], want["lse"])


@pytest.mark.parametrize("n,Lq,sinks", ((6400, 1, 0), (6401, 70, 0), (6463, 33, 65), (6400, 200, 128)))
def test_a_window_of_no_cached_tokens_needs_the_sinks_pages_only(n, Lq, sinks):
    """window 0 without a commit: the table ends with the sinks' pages."""
    Hq, Hkv, D = 4, 2, 128
    pages = -(-sinks // 64)
    table = torch.arange(max(pages, 1), dtype=torch.int32)[None] if pages else torch.full((1, 1), -1, dtype=torch.int32)
    cache = ws.PagedCache.allocate(max(pages, 1), Hkv, D, table, device=DEV, fill_bits=0x7FC1)
    k, v = _randn(1, sinks, Hkv, D), _randn(2, sinks, Hkv, D)
    for page in range(pages):
        m = min(64, sinks - 64 * page)
        cache.k_pool[page, :, :m] = k[64 * page:64 * page + m].transpose(0, 1)
        cache.v_pool[page, :, :m] = v[64 * page:64 * page + m].transpose(0, 1)
    q, kn, vn = _randn(3, 1, Lq, Hq, D), _randn(4, 1, Lq, Hkv, D), _randn(5, 1, Lq, Hkv, D)
    out, lse = ws.block_causal_attn_fwd(q, kn, vn, cache, _pair([n]), window=0, sinks=sinks, want_lse=True)
    at = torch.full((Lq,), sinks, dtype=torch.long)   # the sinks, then the block
    want = ref.attend(q[0], torch.cat([k, kn[0]]), torch.cat([v, vn[0]]), at, at + Lq, sinks, D ** -0.5)
    ref.check("out", out[0], want["out"])
    ref.check("lse", lse[0], want["lse"])


@pytest.mark.parametrize("mistake", ("window + 1", "window - 1", "sinks + 1", "sinks - 1", "block anchor", "none"))
def test_the_bounds_catch_a_shifted_window(mistake):
    """The reference with a planted mistake does not pass (and without one it
    does): one key more or less, or a token-causal token's window counted from
    its block."""
    B, L, H, D, window, sinks = 1, 200, 1, 64, 20, 5
    q, k, v = _randn(1, B, L, H, D), _randn(2, B, L, H, D), _randn(3, B, L, H, D)
    off, starts = [0, 60, 130, L], [40, 130, 150]
    out, lse = ws.block_causal_prefill(q, k, v, _pair([off]), text_starts=_pair([starts]), window=window, sinks=sinks,
                                       want_lse=True, out_dtype=torch.float32)
    lo, hi = ref.ranges(off, starts, window)
    if mistake == "block anchor":
        lo = ref.ranges(off, None, window)[0]
    lo = lo - {"window + 1": 1, "window - 1": -1}.get(mistake, 0)
    s = sinks + {"sinks + 1": 1, "sinks - 1": -1}.get(mistake, 0)
    want = ref.attend(q[0], k[0], v[0], lo, hi, s, D ** -0.5, f32=True)
    wrong = []
    for name, got in (("out", out[0]), ("lse", lse[0])):
        try:
            ref.check(name, got, want[name])
        except AssertionError:
            wrong.append(name)
    assert wrong == ([] if mistake == "none" else ["out", "lse"])
