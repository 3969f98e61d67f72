"""Host and device int32 arrays that the library would misread are refused by
every entry point, through either marshalling, and nothing is written."""
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


def _pair(x):
    h = torch.tensor(x, dtype=torch.int32)
    return h, h.to(DEV)


def bad_pairs(x):
    """Forms of a (host, device) pair whose packed reading is another array, or
    whose copies are not where they are read."""
    h, d = _pair(x)

    def strided(t):
        return torch.stack([t, torch.zeros_like(t)], -1)[..., 0]
    return {"strided host": (strided(h), d), "strided device": (h, strided(d)), "both on the host": (h, h),
            "both on the device": (d, d), "exchanged": (d, h), "int64": (h.long(), d.long()),
            "repeated host": (h[:1].expand(B, *h.shape[1:]), d)}


def _state():
    g = torch.Generator(DEV).manual_seed(1)

    def rnd(*shape):
        return torch.randn(shape, generator=g, device=DEV).to(torch.bfloat16)
    table = torch.arange(8).reshape(2, 4)
    full = ws.PagedCache(rnd(8, HKV, 64, D), rnd(8, HKV, 64, D), table)
    four = ws.PagedCache4.allocate(8, HKV, D, table, device=DEV)
    four.pool.zero_()
    return rnd(B, L, HQ, D), rnd(B, L, HKV, D), rnd(B, L, HKV, D), full, four


FORMS = (
    "strided host", "strided device", "both on the host", "both on the device", "exchanged", "int64", "repeated host")


@pytest.mark.parametrize("native", (True, False))
@pytest.mark.parametrize("form", FORMS)
def test_refused(form, native, monkeypatch):
    gs.say(f"[gpu] int32 arrays: {form}, native={native}")
    q, k, v, full, four = _state()
    lens, off, text = bad_pairs([70, 5])[form], bad_pairs([[0, 2, L]] * 2)[form], bad_pairs([[1, L]] * 2)[form]
    new, starts = bad_pairs([L, 2])[form], bad_pairs([2, 0])[form]
    ok, ok_off = _pair([70, 5]), _pair([[0, 2, L]] * 2)
    out, lse = ws.block_causal_prefill(q, k, v, ok_off, want_lse=True)
    win = dict(window=3, sinks=1)
    calls = {
        "append": lambda: ws.kv_append(full, lens, k, v), "append lens": lambda: ws.kv_append(full, ok, k, v, new_lens=new),
        "append4": lambda: ws.kv_append(four, lens, k, v), "append4 lens": lambda: ws.kv_append(four, ok, k, v, new_lens=new),
        "read4": lambda: ws.kv_read(four, lens, L),
        "step": lambda: ws.block_causal_attn_fwd(q, k, v, full, lens, fuse_append=True),
        "step lens": lambda: ws.block_causal_attn_fwd(q, k, v, full, ok, new_lens=new, fuse_append=True),
        "step text": lambda: ws.block_causal_attn_fwd(q, k, v, full, ok, text_starts=starts, fuse_append=True),
        "noalloc": lambda: ws.block_causal_attn_fwd_noalloc(q, k, v, full, lens, torch.empty_like(q), fuse_append=True),
        "step window": lambda: ws.block_causal_attn_fwd(q, k, v, full, lens, fuse_append=True, **win),
        "step window text": lambda: ws.block_causal_attn_fwd(q, k, v, full, ok, text_starts=starts, fuse_append=True, **win),
        "step4": lambda: ws.block_causal_attn_fwd(q, k, v, four, lens, fuse_append=True),
        "step4 lens": lambda: ws.block_causal_attn_fwd(q, k, v, four, ok, new_lens=new, fuse_append=True),
        "prefill": lambda: ws.block_causal_prefill(q, k, v, off), "prefill paged": lambda: ws.block_causal_prefill(
            q, None, None, off, cache=full),
        "prefill text": lambda: ws.block_causal_prefill(q, k, v, ok_off, text_starts=text),
        "prefill window": lambda: ws.block_causal_prefill(q, k, v, off, **win),
        "gradients": lambda: ws.block_causal_prefill_bwd(q, k, v, out, q, lse, off),
        "gradients window": lambda: ws.block_causal_prefill_bwd(q, k, v, out, q, lse, off, **win),
        "gradients window text": lambda: ws.block_causal_prefill_bwd(q, k, v, out, q, lse, ok_off, text_starts=text, **win),
    }
    ws.library()
    if not native:
        monkeypatch.setattr(ws, "_NATIVE", _Declines())
    before = [t.clone() for t in (full.k_pool, full.v_pool, four.pool)]
    for name, call in calls.items():
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"{name} took {form}")
    torch.cuda.synchronize()
    for x, y in zip((full.k_pool, full.v_pool, four.pool), before):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
