"""Every entry point refuses tensors of another device than the current one (here:
the calls are told that another device is current)."""
import pytest
import torch

import paper_2606_25041_amd as ws
from tests import gpu_support as gs
from tests.test_gpu_argument_tensors import _Declines, caches, pair, rnd

pytestmark = pytest.mark.gpu
B, L, HQ, HKV, D = 2, 5, 4, 2, 64


def test_refused(monkeypatch):
    gs.say("[gpu] another device is current")
    full, four = caches()
    q, k, v, lens, off = rnd(3, B, L, HQ, D), rnd(4, B, L, HKV, D), rnd(5, B, L, HKV, D), pair([70, 5]), pair([[0, L]] * B)
    out, lse = ws.block_causal_prefill(q, k, v, off, want_lse=True)
    torch.cuda.synchronize()
    ws.library()
    calls = (
        lambda: ws.kv_append(full, lens, k, v), lambda: ws.kv_append(four, lens, k, v), lambda: ws.kv_read(four, lens, L),
        lambda: ws.block_causal_attn_fwd(q, k, v, full, lens, out=out), lambda: ws.block_causal_attn_fwd(
            q, k, v, full, lens, window=3, out=out), lambda: ws.block_causal_attn_fwd(q, k, v, four, lens, out=out),
        lambda: ws.block_causal_attn_fwd_noalloc(q, k, v, full, lens, out),
        lambda: ws.block_causal_prefill(q, k, v, off, out=out), lambda: ws.block_causal_prefill(q, k, v, off, window=3, out=out),
        lambda: ws.block_causal_prefill(q, None, None, off, cache=full, out=out),
        lambda: ws.block_causal_prefill_bwd(q, k, v, out, q, lse, off),
        lambda: ws.block_causal_prefill_bwd(q, k, v, out, q, lse, off, window=3))
    with monkeypatch.context() as m:
        m.setattr(ws, "_NATIVE", _Declines())
        m.setattr(torch.cuda, "current_device", lambda: 1)
        for i, call in enumerate(calls):
            with pytest.raises(ValueError, match="current device"):
                call()
                pytest.fail(f"call {i} was taken")
    assert torch.equal(ws.block_causal_prefill(q, k, v, off), out)
