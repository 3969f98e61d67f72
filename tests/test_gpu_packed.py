"""Attention over packed sequences on the GPU: outputs, lse and gradients against
the definition in 64 bits, every element within the bound of the kernels'
roundings (tests/window_ref.py, each sequence on its own)."""
import numpy as np
import pytest
import torch

import paper_2606_25041_amd as ws
from tests import gpu_support as gs
from tests import window_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"


def rnd(seed, *shape):
    g = torch.Generator(DEV).manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).to(torch.bfloat16)


def pair(x):
    h = torch.as_tensor(np.asarray(x), dtype=torch.int32).contiguous()
    return h, h.to(DEV)


def layout(seed, lens, blocks, text):
    """Sequence offsets; with blocks up to that many of each sequence (some
    empty), with text segment starts, as arrays in the packed axis."""
    rng = np.random.default_rng(seed)
    seqs = np.concatenate(([0], np.cumsum(lens)))
    if not blocks:
        return seqs, None, None
    cuts = []
    for a, e in zip(seqs, seqs[1:]):
        cuts += [a, *sorted(rng.integers(a, e + 1, rng.integers(0, blocks)))]
    off = np.array([*cuts, seqs[-1]])
    starts = off[:-1] + (rng.random(len(off) - 1) * (np.diff(off) + 1)).astype(int) if text else None
    return seqs, off, starts


def key_ends(seqs, off, starts, s):
    """lo and hi of the rows of sequence s, counted from its first token."""
    a, e = int(seqs[s]), int(seqs[s + 1])
    i = np.arange(a, e)
    if off is None:
        return np.zeros(e - a, np.int64), i + 1 - a
    n = np.searchsorted(off, i, side="right") - 1
    hi = off[n + 1] if starts is None else np.maximum(starts[n], i + 1)
    return np.zeros(e - a, np.int64), hi - a


CASES = [
    # hq, hkv, d, lens, blocks, text
    (2, 2, 64, [1], 0, False),
    (4, 2, 128, [5, 1, 0, 33, 64, 65, 0], 0, False),
    (8, 1, 64, [256, 257, 255, 1, 700], 0, False),
    (8, 8, 128, [1000, 3, 129, 512], 0, False),
    (3, 1, 128, [90, 300, 0, 17], 4, False),
    (16, 4, 64, [640, 31, 200, 5], 6, True),
    (5, 5, 128, [7] * 60, 0, False),
    (6, 2, 64, [40, 300] * 5, 3, True),
    (1, 1, 128, [2600], 0, False),
]


def inputs(seed, hq, hkv, d, T):
    return rnd(seed, T, hq, d), rnd(seed + 1, T, hkv, d), rnd(seed + 2, T, hkv, d)


@pytest.mark.parametrize("f32", (False, True))
@pytest.mark.parametrize("case", range(len(CASES)))
def test_forward(case, f32):
    hq, hkv, d, lens, blocks, text = CASES[case]
    gs.say(f"[gpu] packed forward {case}: {CASES[case]} f32={f32}")
    seqs, off, starts = layout(case, lens, blocks, text)
    T, tail = int(seqs[-1]), 3 + case % 2 * 200
    q, k, v = inputs(10 * case, hq, hkv, d, T + tail)
    k[T:], v[T:], q[T:] = float("nan"), float("nan"), float("nan")
    out = torch.full((T + tail, hq, d), 7.0, dtype=torch.float32 if f32 else torch.bfloat16, device=DEV)
    lse = torch.full((hq, T + tail), 7.0, device=DEV)
    ws.block_causal_prefill_packed(q, k, v, pair(seqs), None if off is None else pair(off), out=out, lse=lse,
                                   text_starts=None if starts is None else pair(starts))
    torch.cuda.synchronize()
    assert (out[T:] == 7).all() and (lse[:, T:] == 7).all()   # rows behind the last sequence
    for s in range(len(lens)):
        a, e = int(seqs[s]), int(seqs[s + 1])
        lo, hi = key_ends(seqs, off, starts, s)
        if a == e:
            continue
        want = ref.attend(q[a:e], k[a:e], v[a:e], lo, hi, 0, d ** -0.5, f32=f32)
        ref.check(f"out {s}", out[a:e], want["out"])
        ref.check(f"lse {s}", lse[:, a:e], want["lse"])


@pytest.mark.parametrize("bf16", (False, True))
@pytest.mark.parametrize("room", ("full", "least"))
@pytest.mark.parametrize("case", range(len(CASES)))
def test_gradients(case, room, bf16):
    hq, hkv, d, lens, blocks, text = CASES[case]
    gs.say(f"[gpu] packed gradients {case} {room} bf16={bf16}: {CASES[case]}")
    seqs, off, starts = layout(case, lens, blocks, text)
    T, tail = int(seqs[-1]), 5
    q, k, v = inputs(10 * case, hq, hkv, d, T + tail)
    do = rnd(10 * case + 3, T + tail, hq, d)
    kw = dict(text_starts=None if starts is None else pair(starts))
    b = None if off is None else pair(off)
    out, lse = ws.block_causal_prefill_packed(q, k, v, pair(seqs), b, want_lse=True, **kw)
    for x in (q, k, v, do, out):
        x[T:] = float("nan")
    least = -(-8 * hq * (T + tail) // 256) * 256 + 8 * (T + tail)
    dt = torch.bfloat16 if bf16 else torch.float32
    got = [torch.full((T + tail, h, d), 7.0, dtype=dt, device=DEV) for h in (hq, hkv, hkv)]
    call = lambda g, w: ws.block_causal_prefill_packed_bwd(  # noqa: E731
        q, k, v, out, do, lse, pair(seqs), b, dq=g[0], dk=g[1], dv=g[2], workspace=w, **kw)
    space = lambda: torch.empty(least, dtype=torch.uint8, device=DEV) if room == "least" else None  # noqa: E731
    call(got, space())
    again = [torch.full_like(x, 7.0) for x in got]
    call(again, space())
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, again))   # deterministic
    assert all((x[T:] == 7).all() for x in got)
    for s in range(len(lens)):
        a, e = int(seqs[s]), int(seqs[s + 1])
        if a == e:
            continue
        lo, hi = key_ends(seqs, off, starts, s)
        want = ref.attend(q[a:e], k[a:e], v[a:e], lo, hi, 0, d ** -0.5, dout=do[a:e])
        for name, x in zip(("dq", "dk", "dv"), got):
            ref.check(f"{name} {s}", x[a:e], want[name], bf16=bf16)


def test_split_gradients():
    """Few KV heads and one long sequence: its key tiles' rows in shares."""
    gs.say("[gpu] packed gradients, split")
    hq, hkv, d, lens = 8, 1, 64, [20, 3000, 700]
    seqs = np.concatenate(([0], np.cumsum(lens)))
    T = int(seqs[-1])
    q, k, v = inputs(3, hq, hkv, d, T)
    do = rnd(9, T, hq, d)
    out, lse = ws.block_causal_prefill_packed(q, k, v, pair(seqs), want_lse=True)
    got = ws.block_causal_prefill_packed_bwd(q, k, v, out, do, lse, pair(seqs))
    for s in range(3):
        a, e = int(seqs[s]), int(seqs[s + 1])
        lo, hi = key_ends(seqs, None, None, s)
        want = ref.attend(q[a:e], k[a:e], v[a:e], lo, hi, 0, d ** -0.5, dout=do[a:e])
        for name, x in zip(("dq", "dk", "dv"), got):
            ref.check(f"{name} {s}", x[a:e], want[name])


@pytest.mark.parametrize("lens", ([300] * 450, [1] * 140000))
def test_more_tiles_than_a_table(lens):
    """Past 512 items the rows are cut at every 256th token: forward and gradients
    of some sequences against the definition."""
    gs.say(f"[gpu] packed, {len(lens)} sequences")
    hq, hkv, d = 1, 1, 64
    seqs = np.concatenate(([0], np.cumsum(lens)))
    T = int(seqs[-1])
    q, k, v = inputs(5, hq, hkv, d, T)
    do = rnd(8, T, hq, d)
    out, lse = ws.block_causal_prefill_packed(q, k, v, pair(seqs), want_lse=True)
    got = ws.block_causal_prefill_packed_bwd(q, k, v, out, do, lse, pair(seqs))
    for s in (0, 1, 212, 213, len(lens) // 2, len(lens) - 1):
        a, e = int(seqs[s]), int(seqs[s + 1])
        lo, hi = key_ends(seqs, None, None, s)
        want = ref.attend(q[a:e], k[a:e], v[a:e], lo, hi, 0, d ** -0.5, dout=do[a:e])
        ref.check(f"out {s}", out[a:e], want["out"])
        ref.check(f"lse {s}", lse[:, a:e], want["lse"])
        for name, x in zip(("dq", "dk", "dv"), got):
            ref.check(f"{name} {s}", x[a:e], want[name])
    if lens[0] == 1:   # a token alone: its own value
        assert torch.equal(out, v)


def test_a_long_sequence_is_its_own():
    """NaN in one reaches no neighbour of more than 256 tokens, forward or back."""
    gs.say("[gpu] packed, a poisoned sequence")
    hq, hkv, d, lens = 4, 2, 64, [300, 260, 900]
    seqs = np.concatenate(([0], np.cumsum(lens)))
    T = int(seqs[-1])
    q, k, v = inputs(1, hq, hkv, d, T)
    do = rnd(4, T, hq, d)
    clean, lse = ws.block_causal_prefill_packed(q, k, v, pair(seqs), want_lse=True)
    grads = ws.block_causal_prefill_packed_bwd(q, k, v, clean, do, lse, pair(seqs))
    for x in (q, k, v, do):
        x[300:560] = float("nan")
    out, lse2 = ws.block_causal_prefill_packed(q, k, v, pair(seqs), want_lse=True)
    bad = ws.block_causal_prefill_packed_bwd(q, k, v, out, do, lse2, pair(seqs))
    rest = torch.cat((torch.arange(300), torch.arange(560, T))).to(DEV)
    assert out[300:560].isnan().all() and torch.equal(out[rest], clean[rest]) and torch.equal(lse[:, rest], lse2[:, rest])
    for x, y in zip(grads, bad):
        assert torch.equal(x[rest], y[rest])


def test_one_sequence_is_the_whole_prefill():
    """Of one sequence the call is block_causal_prefill, in values."""
    gs.say("[gpu] packed against whole sequences")
    hq, hkv, d, n = 8, 2, 128, 900
    q, k, v = inputs(2, hq, hkv, d, n)
    off = np.array([0, 100, 350, 350, 900])
    whole, lse = ws.block_causal_prefill(q[None], k[None], v[None], pair(off[None]), want_lse=True, out_dtype=torch.float32)
    out, lse2 = ws.block_causal_prefill_packed(q, k, v, pair([0, n]), pair(off), want_lse=True, out_dtype=torch.float32)
    # (the whole prefill's weights are one bf16, half a step off: 2^-8 of the sum of |weight x value|, below 4 here)
    assert (out - whole[0]).abs().max() < 2 * 2 ** -8 * 4 and (lse[0] - lse2).abs().max() < 1e-5


def test_layouts():
    """Views into one fused projection, outputs into views: bit for bit."""
    gs.say("[gpu] packed, layouts")
    hq, hkv, d, lens = 4, 2, 64, [70, 300, 9]
    seqs = pair(np.concatenate(([0], np.cumsum(lens))))
    T = sum(lens)
    fused = rnd(1, T, hq + 2 * hkv, d)
    q, k, v = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
    do = rnd(2, T, hq, d)
    plain, lse = ws.block_causal_prefill_packed(q.contiguous(), k.contiguous(), v.contiguous(), seqs, want_lse=True)
    wide = torch.full((T, 2 * hq, d), 7.0, dtype=torch.bfloat16, device=DEV)
    ws.block_causal_prefill_packed(q, k, v, seqs, out=wide[:, 1::2])
    assert torch.equal(wide[:, 1::2], plain) and (wide[:, ::2] == 7).all()
    grads = ws.block_causal_prefill_packed_bwd(q.contiguous(), k.contiguous(), v.contiguous(), plain, do, lse, seqs)
    dfused = torch.zeros(T, hq + 2 * hkv, d, device=DEV)
    ws.block_causal_prefill_packed_bwd(q, k, v, wide[:, 1::2], do, lse, seqs, dq=dfused[:, :hq], dk=dfused[:, hq:hq + hkv],
                                       dv=dfused[:, hq + hkv:])
    assert torch.equal(dfused, torch.cat(grads, 1))
