"""What is not finite stays in its own sequence of a packed call, also past the tables
of a launch (512 items of rows, 320 of keys).  Everything of the other sequences, outputs,
log-sum-exps and gradients, is what it is without it, bit for bit; what sees it is
not finite."""
import numpy as np
import pytest
import torch

import paper_2606_25041_amd as ws
from tests import gpu_support as gs

pytestmark = pytest.mark.gpu
DEV = "cuda"
NAN, INF = float("nan"), float("inf")


def rnd(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV).to(torch.bfloat16)


def pair(x):
    h = torch.as_tensor(np.asarray(x), dtype=torch.int32).contiguous()
    return h, h.to(DEV)


def calls(q, k, v, do, seqs, blocks, text, f32, bf16):
    kw = dict(text_starts=text)
    if f32:
        out, lse = ws.block_causal_prefill_packed(q, k, v, seqs, blocks, want_lse=True, out_dtype=torch.float32, **kw)
    else:
        out, lse = ws.block_causal_prefill_packed(q, k, v, seqs, blocks, want_lse=True, **kw)
    grads = ws.block_causal_prefill_packed_bwd(q, k, v, out.to(torch.bfloat16), do, lse, seqs, blocks,
                                               grad_dtype=torch.bfloat16 if bf16 else torch.float32, **kw)
    return [out, lse.T.contiguous(), *grads]


def check(hq, hkv, d, lens, bad, blocks=None, text=None, f32=False, bf16=False, poison=(("q", NAN), ("k", NAN), ("v", NAN), ("do", NAN))):
    """Sequence `bad` has one bad element in the middle; all others stay as they were."""
    seqs = np.concatenate(([0], np.cumsum(lens)))
    T, (a, e) = int(seqs[-1]), seqs[bad:bad + 2].tolist()
    x = {"q": rnd(1, T, hq, d), "k": rnd(2, T, hkv, d), "v": rnd(3, T, hkv, d), "do": rnd(4, T, hq, d)}
    ends = None if blocks is None else pair(blocks)
    starts = None if text is None else pair(text)
    clean = calls(*x.values(), pair(seqs), ends, starts, f32, bf16)
    assert all(t.isfinite().all() for t in clean)
    rest = torch.cat((torch.arange(a), torch.arange(e, T))).to(DEV)
    at, dim, g = (a + e) // 2, 3, hq // hkv
    for name, value in poison:
        gs.say(f"[gpu] packed, {value} in {name} of sequence {bad} of {len(lens)} ({lens[:6]}..), {hq}/{hkv} x {d} f32={f32} bf16={bf16}")
        y = dict(x)
        y[name] = x[name].clone()
        y[name][at, 0, dim] = value
        got = calls(*y.values(), pair(seqs), ends, starts, f32, bf16)
        for what, p, c in zip(("out", "lse", "dq", "dk", "dv"), got, clean):
            same = torch.equal(p[rest], c[rest])
            assert same, (name, value, what, (p[rest] != c[rest]).nonzero()[:4].tolist())
        out, lse, dq, dk, dv = got
        # (of infinite scores only some are not finite)
        if name == "q" and value != value:
            assert not out[at, 0].isfinite().any() and not lse[at, 0].isfinite()
        elif name == "k" and value != value:
            assert not out[at:e, :g].isfinite().any() if blocks is None else not out[at, :g].isfinite().any()
            assert not dq[at, :g].isfinite().any() and not dk[at, 0].isfinite().any()
        elif name == "v":
            # the rows that see it, in its head dim
            assert not out[at:e, :g, dim].isfinite().any() and not dq[at, :g].isfinite().any()
        elif name == "do":
            # (its token's query sees itself, and every key before it)
            assert not dv[a:at + 1, 0, dim].isfinite().any() and not dq[at, 0].isfinite().any()


@pytest.mark.parametrize("lens,bad", (([260] * 107, 50), ([260] * 171, 80), ([20500, 20500], 0), ([20500, 20500], 1), ([700] * 58, 29)))
def test_past_the_tables_of_the_gradients(lens, bad):
    """More key or row items than a launch's table holds: tiles of any neighbours."""
    check(2, 1, 64, lens, bad, bf16=True)
