"""An lse of another type or layout is refused by every entry point that takes
one, through either marshalling, and nothing is written."""
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


@pytest.mark.parametrize("native", (True, False))
@pytest.mark.parametrize("form", ("bf16", "f64", "transposed", "repeated"))
def test_refused(form, native, monkeypatch):
    gs.say(f"[gpu] lse: {form}, native={native}")
    g = torch.Generator(DEV).manual_seed(1)

    def rnd(*shape):
        return torch.randn(shape, generator=g, device=DEV).to(torch.bfloat16)

    def pair(x):
        h = torch.tensor(x, dtype=torch.int32)
        return h, h.to(DEV)
    q, k, v = rnd(B, L, HQ, D), rnd(B, L, HKV, D), rnd(B, L, HKV, D)
    table = torch.arange(8).reshape(2, 4)
    full = ws.PagedCache(rnd(8, HKV, 64, D), rnd(8, HKV, 64, D), table)
    four = ws.PagedCache4.allocate(8, HKV, D, table, device=DEV)
    four.pool.zero_()
    lens, off = pair([70, 5]), pair([[0, 2, L]] * 2)
    out, good = ws.block_causal_prefill(q, k, v, off, want_lse=True)
    bad = {"bf16": good.to(torch.bfloat16), "f64": good.double(),
           "transposed": torch.zeros(B, L, HQ, device=DEV).transpose(1, 2),
           "repeated": torch.zeros(1, HQ, L, device=DEV).expand(B, HQ, L)}[form]
    ws.library()
    if not native:
        monkeypatch.setattr(ws, "_NATIVE", _Declines())
    win = dict(window=3)
    before = bad.clone()
    for i, call in enumerate((
            lambda: ws.block_causal_attn_fwd(q, k, v, full, lens, lse=bad),
            lambda: ws.block_causal_attn_fwd(q, k, v, full, lens, lse=bad, **win),
            lambda: ws.block_causal_attn_fwd(q, k, v, four, lens, lse=bad, want_lse=True),
            lambda: ws.block_causal_attn_fwd_noalloc(q, k, v, full, lens, torch.empty_like(q), lse=bad),
            lambda: ws.block_causal_prefill(q, k, v, off, lse=bad),
            lambda: ws.block_causal_prefill(q, k, v, off, lse=bad, **win),
            lambda: ws.block_causal_prefill_bwd(q, k, v, out, q, bad, off),
            lambda: ws.block_causal_prefill_bwd(q, k, v, out, q, bad, off, **win))):
        with pytest.raises(ValueError, match="f32"):
            call()
            pytest.fail(f"call {i} took {form}")
    torch.cuda.synchronize()
    assert torch.equal(bad, before)
