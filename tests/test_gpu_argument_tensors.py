"""Tensors whose memory a kernel must not be given (on the host, strided where
the library takes packed ones) are refused by every entry point, through either
marshalling, and nothing is written."""
import pytest
import torch

import paper_2606_25041_amd as ws
from tests import gpu_support as gs

pytestmark = pytest.mark.gpu
DEV = "cuda"
B, L, HQ, HKV, D = 2, 5, 4, 2, 64


class _Declines:
    """Takes no call, so every call goes through the Python code."""

    def __getattr__(self, name):
        return lambda *_: None


def rnd(seed, *shape):
    g = torch.Generator(DEV).manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).to(torch.bfloat16)


def pair(x):
    h = torch.tensor(x, dtype=torch.int32)
    return h, h.to(DEV)


def caches():
    table = torch.arange(8).reshape(2, 4)
    four = ws.PagedCache4.allocate(8, HKV, D, table, device=DEV)
    four.pool.zero_()
    return ws.PagedCache(rnd(1, 8, HKV, 64, D), rnd(2, 8, HKV, 64, D), table), four


CACHE_FORMS = ("pools on the host", "table on the host", "strided pools", "bytes for bf16", "64-bit table", "strided table")


def spoil(cache, form):
    names = ("pool",) if isinstance(cache, ws.PagedCache4) else ("k_pool", "v_pool")
    for n in names:
        p = getattr(cache, n)
        if form == "pools on the host":
            setattr(cache, n, p.cpu())
        elif form == "strided pools":
            setattr(cache, n, torch.cat((p, p), -1)[..., :p.shape[-1]])
        elif form == "bytes for bf16":
            setattr(cache, n, torch.zeros(p.shape, dtype=torch.int8 if len(names) > 1 else torch.int16, device=DEV))
    if form == "table on the host":
        cache.page_table = cache.page_table_host
    elif form == "64-bit table":
        cache.page_table, cache.page_table_host = cache.page_table.long(), cache.page_table_host.long()
    elif form == "strided table":
        h = torch.stack((cache.page_table_host,) * 2, -1)
        cache.page_table_host, cache.page_table = h[..., 0], h.to(DEV)[..., 0]
    return cache


def refused(calls, native, monkeypatch):
    ws.library()
    if not native:
        monkeypatch.setattr(ws, "_NATIVE", _Declines())
    for i, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was taken")
    torch.cuda.synchronize()


@pytest.mark.parametrize("native", (True, False))
@pytest.mark.parametrize("form", CACHE_FORMS)
def test_caches(form, native, monkeypatch):
    gs.say(f"[gpu] caches: {form}, native={native}")
    full, four = (spoil(c, form) for c in caches())
    q, k, v, lens, off = rnd(3, B, L, HQ, D), rnd(4, B, L, HKV, D), rnd(5, B, L, HKV, D), pair([70, 5]), pair([[0, L]] * B)
    refused((
        lambda: ws.kv_append(full, lens, k, v),
        lambda: ws.kv_append(four, lens, k, v),
        lambda: ws.kv_read(four, lens, L),
        lambda: ws.block_causal_attn_fwd(q, k, v, full, lens),
        lambda: ws.block_causal_attn_fwd(q, k, v, full, lens, window=3),
        lambda: ws.block_causal_attn_fwd(q, k, v, four, lens),
        lambda: ws.block_causal_attn_fwd_noalloc(q, k, v, full, lens, torch.empty_like(q)),
        lambda: ws.block_causal_prefill(q, None, None, off, cache=full),
        lambda: ws.block_causal_prefill(q, None, None, off, cache=full, window=3),
    ), native, monkeypatch)


@pytest.mark.parametrize("native", (True, False))
@pytest.mark.parametrize("form", ("query", "workspace", "strided workspace"))
def test_queries_and_workspaces(form, native, monkeypatch):
    gs.say(f"[gpu] {form} on the host, native={native}")
    full, four = caches()
    q, k, v, lens, off = rnd(3, B, L, HQ, D), rnd(4, B, L, HKV, D), rnd(5, B, L, HKV, D), pair([70, 5]), pair([[0, L]] * B)
    out, lse = ws.block_causal_prefill(q, k, v, off, want_lse=True)
    use, host = {}, torch.zeros(1 << 20, dtype=torch.uint8)
    if form == "query":
        q = q.cpu()
    else:
        use = dict(workspace=host if form == "workspace" else host.to(DEV)[::2])
    calls = [
        lambda: ws.block_causal_attn_fwd(q, k, v, full, lens, out=torch.empty_like(out), **use),
        lambda: ws.block_causal_attn_fwd(q, k, v, full, lens, window=3, out=torch.empty_like(out), **use),
        lambda: ws.block_causal_attn_fwd(q, k, v, four, lens, out=torch.empty_like(out), **use),
        lambda: ws.block_causal_prefill_bwd(q, k, v, out, out, lse, off, **use),
        lambda: ws.block_causal_prefill_bwd(q, k, v, out, out, lse, off, window=3, **use),
    ]
    if form == "query":
        calls += [
            lambda: ws.block_causal_attn_fwd_noalloc(q, k, v, full, lens, torch.empty_like(out)),
            lambda: ws.block_causal_prefill(q, k, v, off, out=torch.empty_like(out)),
            lambda: ws.block_causal_prefill(q, k, v, off, window=3, out=torch.empty_like(out)),
        ]
    refused(calls, native, monkeypatch)
