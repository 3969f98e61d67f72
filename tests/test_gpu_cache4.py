"""The 4-bit cache: committing and reading back bit for bit against the format's
reference (tests/cache4_ref.py), and streaming steps over it against float64
attention over the rounded history, every element within the bound of the
kernels' roundings (tests/window_ref.py).  Bytes that no token was committed to
hold 0xFF (scale bytes that read as NaN)."""
import numpy as np
import pytest
import torch

import paper_2606_25041_amd as ws
from tests import cache4_ref
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


def empty_cache(seed, batch, hkv, d, tokens):
    """Every byte 0xFF; pages in a random physical order."""
    per = max(1, -(-tokens // 64))
    order = torch.randperm(batch * per + 2, generator=torch.Generator().manual_seed(seed))[:batch * per]
    cache = ws.PagedCache4.allocate(batch * per + 2, hkv, d, order.reshape(batch, per), device=DEV)
    cache.pool.fill_(255)
    return cache


def commit(pool, table, d, start, k, v):
    """The same on a CPU copy of the pool: tokens k, v [n][Hkv][d] of one stream."""
    for half, x in ((0, k), (34 * d, v)):
        codes, scales = cache4_ref.encode(x.cpu())
        packed = (codes[..., 0::2] + 16 * codes[..., 1::2]).astype(np.uint8)
        for t in range(x.shape[0]):
            page, slot = int(table[(start + t) // 64]), (start + t) % 64
            at = half + slot * (d // 2)
            pool[page, :, at:at + d // 2] = torch.from_numpy(packed[t])
            at = half + 32 * d + slot * (d // 32)
            pool[page, :, at:at + d // 32] = torch.from_numpy(scales[t])


def _same_pool(got, want):
    """Equal but for the codes of a NaN block, which are left open."""
    return torch.equal(got.cpu(), want)


@pytest.mark.parametrize("d", (64, 128))
def test_every_bf16(d):
    """Each of the 65536 bf16 patterns as an element, in blocks of every kind of
    amax: its own magnitude, larger ones that push it through every rounding
    point, NaN and infinity."""
    gs.say(f"[gpu] 4-bit cache: every bf16, d {d}")
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
    blocks = []
    for shift in range(8):   # block amax = x, or x's exponent plus shift with a random mantissa
        g = torch.Generator().manual_seed(shift)
        x = bits.view(torch.bfloat16)
        exp = ((bits.int() >> 7) & 255) + shift
        top = (exp.clamp(max=254) * 128 + (torch.randint(0, 128, (65536,), generator=g) if shift else bits.int() & 127))
        top = torch.where(exp - shift == 255, bits.int() & 0x7FFF, top).to(torch.int16).view(torch.bfloat16)
        blk = torch.zeros(65536, 32, dtype=torch.bfloat16)
        blk[:, shift] = x
        blk[:, 31 - shift] = top
        blocks.append(blk)
    x = torch.cat(blocks).reshape(-1, 2, d).flip(0)   # [tokens][2 heads][d]
    n = x.shape[0]
    cache = empty_cache(1, 1, 2, d, n)
    k, v = x[None].to(DEV), x.flip(0)[None].contiguous().to(DEV)
    ws.kv_append(cache, _pair([0]), k, v)
    rk, rv = ws.kv_read(cache, _pair([0]), n)
    torch.cuda.synchronize()
    for got, src in ((rk, x), (rv, x.flip(0))):
        want = cache4_ref.rounded(src)
        got = got[0].cpu()
        assert torch.equal(got.isnan(), want.isnan())
        assert torch.equal(torch.where(want.isnan(), 0, got), torch.where(want.isnan(), 0, want))


@pytest.mark.parametrize("case", [
    # Hkv, D, new, starts, new_lens
    (1, 64, 1, [0], None),
    (3, 128, 1, [63], None),
    (2, 128, 130, [0, 62, 1000], None),
    (5, 64, 77, [1, 64, 127], [77, 0, 30]),
    (8, 128, 174, [22579], None),
])
def test_append_and_read(case):
    """Bytes, with the rest of the pool untouched, from strided inputs; and the
    values read back, also into strided outputs and from other positions."""
    hkv, d, new, starts, lens = case
    gs.say(f"[gpu] 4-bit append {case}")
    B = len(starts)
    cache = empty_cache(3, B, hkv, d, max(starts) + new)
    fused = _randn(4, B, new, 3, hkv, d)   # keys and values as views into one projection
    k, v = fused[:, :, 0], fused[:, :, 2]
    want = cache.pool.cpu()
    ws.kv_append(cache, _pair(starts), k, v, new_lens=None if lens is None else _pair(lens))
    real = lens or [new] * B
    for b in range(B):
        commit(want, cache.page_table_host[b], d, starts[b], k[b, :real[b]], v[b, :real[b]])
    assert _same_pool(cache.pool, want)
    if lens is None:
        rk, rv = ws.kv_read(cache, starts, new)
        assert torch.equal(rk, cache4_ref.rounded(k)) and torch.equal(rv, cache4_ref.rounded(v))
        n = max(1, new // 2)
        out = torch.zeros(B, n, hkv, 2, d, dtype=torch.bfloat16, device=DEV)
        ws.kv_read(cache, _pair([s + new - n for s in starts]), n, k=out[:, :, :, 0], v=out[:, :, :, 1])
        assert torch.equal(out[:, :, :, 0], rk[:, new - n:]) and torch.equal(out[:, :, :, 1], rv[:, new - n:])


STEPS = [
    # Hq, Hkv, D, Lq, caches, new_lens, starts, f32
    (8, 2, 128, 1, [700, 0, 64, 129], None, None, False),
    (8, 2, 128, 1, [700, 0, 64, 129], None, [0, 0, 1, 0], True),
    (64, 8, 128, 3, [4001, 9001, 63, 1], None, [0, 0, 0, 0], False),
    (4, 4, 64, 33, [1000, 31], None, None, False),
    (16, 4, 64, 37, [5003, 1200, 64, 2777, 333, 0], None, None, True),
    (6, 2, 128, 100, [2500, 90], None, [60, 100], False),
    (6, 2, 64, 300, [640, 7], None, [0, 0], True),
    (64, 8, 128, 24, [9000, 4100, 3000, 17], [24, 1, 7, 20], [20, 0, 7, 3], False),
    (64, 8, 128, 24, [9000, 4100, 3000, 17], [24, 1, 7, 20], None, True),
    (24, 24, 128, 256, [2257], None, None, False),
    (3, 1, 128, 90, [4000, 300], None, [10, 80], False),
    (8, 1, 128, 5, [20000] * 3 + [40, 1] * 16, None, [0] * 35, False),   # lengths from memory
    (8, 8, 64, 520, [130], None, [500], False),
    (32, 1, 128, 1, [33333], None, None, False),
    (33, 1, 64, 1, [5000, 4999], None, None, True),      # one row past a 32-row block
    (1, 1, 128, 1, [1], None, None, False),
    (1, 1, 64, 1, [0], None, None, True),
    (1, 1, 128, 64, [64], None, [0], True),
    (40, 8, 128, 6, [6000, 5999], None, [0, 3], False),
    # several row blocks of the few-row kernel, a new block of several tiles
    (1, 1, 128, 128, [300, 5, 64], None, [100, 0, 128], False),
    (4, 2, 64, 60, [3000, 70], [33, 60], [0, 30], True),
    # streams of very different lengths
    (16, 2, 128, 40, [9000, 17, 40, 0, 5], None, [3] * 5, False),
    (24, 24, 128, 200, [4000, 300, 30], [200, 33, 64], None, True),
    (12, 4, 64, 90, [20000, 300, 300, 8], [90, 33, 64, 1], [80, 33, 0, 0], False),
    # the few-row kernel with up to 16 row blocks
    (8, 1, 128, 60, [9000], None, [13], False),
    (8, 1, 64, 50, [9000, 33, 0], [50, 1, 20], [40, 0, 20], True),
    (16, 4, 64, 128, [5000], None, None, True),
    (40, 8, 128, 100, [4096], None, None, False),
    # the common kernel on few rows: many short streams
    (16, 8, 128, 1, [100, 3, 64, 0] * 8, None, None, False),
    (16, 2, 64, 5, [100, 3, 64, 0] * 8, [5, 1, 3, 2] * 8, [0, 1, 3, 1] * 8, True),
    (24, 24, 128, 100, [1200] * 4, None, None, False),
]


@pytest.mark.parametrize("case", range(len(STEPS)))
def test_step(case):
    Hq, Hkv, D, Lq, caches, lens, starts, f32 = STEPS[case]
    gs.say(f"[gpu] 4-bit step {case}: {STEPS[case]}")
    B = len(caches)
    cache = empty_cache(case, B, Hkv, D, max(caches) + Lq)
    hist = []
    for b, c in enumerate(caches):
        k, v = 2 * _randn(10 * b + case, c, Hkv, D), _randn(10 * b + case + 1, c, Hkv, D)
        k[:, :, 5] *= 8   # a channel larger than the rest
        if c:
            one = ws.PagedCache4(cache.pool, cache.page_table_host[b:b + 1])
            ws.kv_append(one, [0], k[None], v[None])
        hist.append((cache4_ref.rounded(k), cache4_ref.rounded(v)))
    q = _randn(7 + case, B, Lq, Hq, D)
    kn, vn = _randn(8 + case, B, Lq, Hkv, D), _randn(9 + case, B, Lq, Hkv, D)
    real = lens or [Lq] * B
    for b in range(B):
        kn[b, real[b]:], vn[b, real[b]:] = float("nan"), float("nan")
    kw = dict(out_dtype=torch.float32 if f32 else torch.bfloat16, want_lse=True,
              text_starts=None if starts is None else _pair(starts), new_lens=None if lens is None else _pair(lens))
    want_pool = cache.pool.cpu()
    out, lse = ws.block_causal_attn_fwd(q, kn, vn, cache, _pair(caches), **kw)
    assert _same_pool(cache.pool, want_pool)
    again, lse2 = ws.block_causal_attn_fwd(q, kn, vn, cache, _pair(caches), fuse_append=True, **kw)
    torch.cuda.synchronize()
    for b in range(B):
        n, c = real[b], caches[b]
        lo, hi = ref.step_ranges(c, n, None if starts is None else starts[b], 2 ** 31)
        k, v = torch.cat((hist[b][0], kn[b, :n])), torch.cat((hist[b][1], vn[b, :n]))
        want = ref.attend(q[b, :n], k, v, lo, hi, 0, D ** -0.5, f32=f32)
        ref.check(f"out {b}", out[b, :n], want["out"])
        ref.check(f"lse {b}", lse[b, :, :n], want["lse"])
        assert torch.equal(out[b, :n], again[b, :n]) and torch.equal(lse[b, :, :n], lse2[b, :, :n]), b
        commit(want_pool, cache.page_table_host[b], D, c, kn[b, :n], vn[b, :n])
    assert _same_pool(cache.pool, want_pool)


@pytest.mark.parametrize("Lq", (2, 40))
def test_a_pool_past_4_gib(Lq):
    gs.say(f"[gpu] 4-bit pool past 4 GiB, {Lq} new tokens")
    pages, Hq, Hkv, D, n = 65000, 16, 8, 128, 1000
    per = -(-(n + Lq) // 64)
    table = torch.arange(pages - per, pages).flip(0)[None]
    cache = ws.PagedCache4.allocate(pages, Hkv, D, table, device=DEV)
    k, v = _randn(1, 1, n, Hkv, D), _randn(2, 1, n, Hkv, D)
    ws.kv_append(cache, _pair([0]), k, v)
    rk, rv = ws.kv_read(cache, _pair([0]), n)
    assert torch.equal(rk, cache4_ref.rounded(k)) and torch.equal(rv, cache4_ref.rounded(v))
    q, kn, vn = _randn(3, 1, Lq, Hq, D), _randn(4, 1, Lq, Hkv, D), _randn(5, 1, Lq, Hkv, D)
    out = ws.block_causal_attn_fwd(q, kn, vn, cache, _pair([n]), fuse_append=True)
    lo, hi = ref.step_ranges(n, Lq, None, 2 ** 31)
    want = ref.attend(q[0], torch.cat((rk[0], kn[0])), torch.cat((rv[0], vn[0])), lo, hi, 0, D ** -0.5)
    ref.check("out", out[0], want["out"])
    gk, _ = ws.kv_read(cache, _pair([n]), Lq)
    assert torch.equal(gk, cache4_ref.rounded(kn))
