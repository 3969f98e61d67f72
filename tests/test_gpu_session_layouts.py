"""The windowed and 4-bit calls on strided tensors (views into one projection,
heads before tokens, a batch that repeats one sequence, rows far apart) and with
outputs and gradients in views of larger buffers: bit for bit the contiguous
calls, and nothing else written."""
import pytest
import torch

import paper_2606_25041_amd as ws
from tests import gpu_support as gs
from tests.test_gpu_argument_tensors import pair, rnd

pytestmark = pytest.mark.gpu
DEV = "cuda"
HQ, HKV = 8, 2
LAYOUTS = ("projection", "heads first", "one sequence", "far apart")


def tensors(layout, B, L, d, *heads):
    """Random [B][L][h][d] tensors of a layout."""
    if layout == "projection":
        return rnd(1, B, L, sum(heads), d).split(heads, 2)
    if layout == "heads first":
        return [rnd(i, B, h, L, d).transpose(1, 2) for i, h in enumerate(heads)]
    if layout == "one sequence":
        return [rnd(i, 1, L, h, d).expand(B, L, h, d) for i, h in enumerate(heads)]
    out = []   # (queries and upstream gradients: 2^24 elements and more; keys and values: just below)
    for i, h in enumerate(heads):
        step = 2 ** 24 + 8 if h == HQ else 2 ** 24 - 8
        t = torch.empty((B * L - 1) * step + h * d, dtype=torch.bfloat16, device=DEV).as_strided((B, L, h, d), (L * step, step, d, 1))
        out.append(t.copy_(rnd(i, B, L, h, d)))
    return out


class Buffers:
    """Outputs in views of larger buffers, whose other elements must stay."""

    def __init__(self):
        self.all = []

    def view(self, B, L, H, d, dtype):
        whole = torch.full((B, L + 1, H + 3, d + 8), 7.0, dtype=dtype, device=DEV)
        view = whole[:, :L, 2:2 + H, :d]
        self.all.append((whole, view))
        return view

    def untouched(self):
        for whole, view in self.all:
            view.fill_(7.0)
            assert bool((whole == 7.0).all())


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.parametrize("f32", (False, True))
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("new", (2, 40))
@pytest.mark.parametrize("four", (False, True))
def test_steps(four, new, layout, d, f32):
    gs.say(f"[gpu] strided steps: four={four} new={new} {layout} d={d} f32={f32}")
    B, caches = 2, [700, 130]
    per = -(-(max(caches) + new) // 64)
    table = torch.arange(B * per).flip(0).reshape(B, per)

    def cache():
        if four:
            c = ws.PagedCache4.allocate(B * per, HKV, d, table, device=DEV)
            c.pool.zero_()
            ws.kv_append(c, pair([0, 0]), rnd(8, B, 700, HKV, d), rnd(9, B, 700, HKV, d), new_lens=pair(caches))
            return c
        return ws.PagedCache(rnd(8, B * per, HKV, 64, d), rnd(9, B * per, HKV, 64, d), table)
    q, k, v = tensors(layout, B, new, d, HQ, HKV, HKV)
    dtype, buf, win = torch.float32 if f32 else torch.bfloat16, Buffers(), {} if four else dict(window=300, sinks=65)
    a, b, out = cache(), cache(), buf.view(B, new, HQ, d, dtype)
    _, lse = ws.block_causal_attn_fwd(q, k, v, a, pair(caches), out=out, want_lse=True, fuse_append=True, **win)
    want, wl = ws.block_causal_attn_fwd(q.contiguous(), k.contiguous(), v.contiguous(), b, pair(caches), out_dtype=dtype,
                                        want_lse=True, fuse_append=True, **win)
    torch.cuda.synchronize()
    assert same(out, want) and torch.equal(lse, wl)
    for name in ("pool",) if four else ("k_pool", "v_pool"):
        assert same(getattr(a, name), getattr(b, name))
    buf.untouched()
    ws.kv_append(a, pair([5, 64]), k, v)
    ws.kv_append(b, pair([5, 64]), k.contiguous(), v.contiguous())
    for name in ("pool",) if four else ("k_pool", "v_pool"):
        assert same(getattr(a, name), getattr(b, name))
    if four:
        rk, rv = buf.view(B, new, HKV, d, torch.bfloat16), buf.view(B, new, HKV, d, torch.bfloat16)
        ws.kv_read(a, pair([5, 64]), new, k=rk, v=rv)
        wk, wv = ws.kv_read(b, pair([5, 64]), new)
        assert same(rk, wk) and same(rv, wv)
        buf.untouched()


@pytest.mark.parametrize("bf16", (False, True))
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("layout", LAYOUTS)
def test_prefill_and_gradients(layout, d, bf16):
    gs.say(f"[gpu] strided prefill and gradients: {layout} d={d} bf16={bf16}")
    B, L = 2, 70 if layout == "far apart" else 333
    off, text = pair([[0, 20, 20, 65, L], [0, 1, 2, 60, L]]), pair([[20, 20, 40, L], [0, 2, 60, 66]])
    win = dict(text_starts=text, window=30, sinks=9)
    q, k, v = tensors(layout, B, L, d, HQ, HKV, HKV)
    do, = tensors(layout, B, L, d, HQ)
    qc, kc, vc, dc = (x.contiguous() for x in (q, k, v, do))
    buf = Buffers()
    for f32 in (True, False):
        out = buf.view(B, L, HQ, d, torch.float32 if f32 else torch.bfloat16)
        _, lse = ws.block_causal_prefill(q, k, v, off, out=out, want_lse=True, **win)
        want, wl = ws.block_causal_prefill(qc, kc, vc, off, out_dtype=out.dtype, want_lse=True, **win)
        assert same(out, want) and torch.equal(lse, wl)
    grad = torch.bfloat16 if bf16 else torch.float32
    dq, dk, dv = buf.view(B, L, HQ, d, grad), buf.view(B, L, HKV, d, grad), buf.view(B, L, HKV, d, grad)
    ws.block_causal_prefill_bwd(q, k, v, out, do, lse, off, dq=dq, dk=dk, dv=dv, **win)
    ref = ws.block_causal_prefill_bwd(qc, kc, vc, want, dc, wl, off, grad_dtype=grad, **win)
    torch.cuda.synchronize()
    assert all(same(x, y) for x, y in zip((dq, dk, dv), ref))
    buf.untouched()
