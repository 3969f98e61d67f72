"""Workspaces that the caller brings, of the sizes that the Python queries give:
enough for every windowed and 4-bit call, one byte less refused, and the same
results as with the call's own."""
import pytest
import torch

import paper_2606_25041_amd as ws
from tests import gpu_support as gs
from tests.test_gpu_argument_tensors import pair, rnd

pytestmark = pytest.mark.gpu
DEV = "cuda"
HQ, HKV, D, CACHES = 8, 2, 128, [3000, 700]
PER = -(-(max(CACHES) + 200) // 64)


def _both(need, call):
    assert need > 0
    want = call(None)
    got = call(torch.empty(need, dtype=torch.uint8, device=DEV))
    with pytest.raises(ws.WsError, match="workspace"):
        call(torch.empty(need - 1, dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("lens", (None, [150, 90]))
@pytest.mark.parametrize("new", (2, 150))
def test_steps(new, lens):
    gs.say(f"[gpu] own workspaces, {new} new tokens")
    lens = None if lens is None else [min(x, new) for x in lens]
    table = torch.arange(2 * PER).reshape(2, PER)
    full = ws.PagedCache(rnd(1, 2 * PER, HKV, 64, D), rnd(2, 2 * PER, HKV, 64, D), table)
    four = ws.PagedCache4.allocate(2 * PER, HKV, D, table, device=DEV)
    ws.kv_append(four, pair([0, 0]), rnd(3, 2, 3000, HKV, D), rnd(4, 2, 3000, HKV, D))
    q, k, v = rnd(5, 2, new, HQ, D), rnd(6, 2, new, HKV, D), rnd(7, 2, new, HKV, D)
    kw = dict(new_lens=None if lens is None else pair(lens))
    real = lens or [new] * 2

    def step(cache, **win):
        def call(workspace):
            out = ws.block_causal_attn_fwd(q, k, v, cache, pair(CACHES), workspace=workspace, **kw, **win)
            return [out[b, :n] for b, n in enumerate(real)]
        return call
    shape = (2, HQ, HKV, new, CACHES, lens)
    _both(ws.step_workspace_bytes_window(*shape, sinks=65, window=2000), step(full, sinks=65, window=2000))
    _both(ws.step_workspace_bytes_4bit(*shape), step(four))


def test_gradients():
    gs.say("[gpu] own workspaces, gradients")
    L, sinks, window = 900, 5, 200
    q, k, v, do = rnd(1, 1, L, HQ, D), rnd(2, 1, L, HKV, D), rnd(3, 1, L, HKV, D), rnd(4, 1, L, HQ, D)
    off = pair([[0, 200, 450, L]])
    win = dict(window=window, sinks=sinks)
    out, lse = ws.block_causal_prefill(q, k, v, off, want_lse=True, **win)
    need = ws.prefill_window_bwd_workspace_bytes(1, HQ, HKV, L, sinks, window)
    want = ws.block_causal_prefill_bwd(q, k, v, out, do, lse, off, **win)
    got = ws.block_causal_prefill_bwd(q, k, v, out, do, lse, off, workspace=torch.empty(need, dtype=torch.uint8, device=DEV), **win)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    with pytest.raises(ws.WsError, match="workspace"):
        ws.block_causal_prefill_bwd(q, k, v, out, do, lse, off, workspace=torch.empty(64, dtype=torch.uint8, device=DEV), **win)
    with pytest.raises(ValueError):
        ws.prefill_window_bwd_workspace_bytes(1, HQ, HKV, L, -1, window)
