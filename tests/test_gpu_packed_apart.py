"""What is not finite stays in its own sequence of a packed call, at any lengths: of
neighbours that share a work-group's rows or keys, and past the tables of a launch
(512 items of rows, 320 of keys).  Everything of the other sequences, outputs,
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


SHORT = [5, 33, 1, 64, 100, 20, 0, 30, 3]
ALL = tuple((n, v) for n in ("q", "k", "v", "do") for v in (NAN, INF, -INF))


@pytest.mark.parametrize("f32,bf16", ((False, True), (True, False)))
@pytest.mark.parametrize("hq,hkv,d", ((4, 2, 64), (2, 2, 128), (8, 1, 128)))
@pytest.mark.parametrize("bad", (0, 1, 4, 8))
def test_short_neighbours(hq, hkv, d, bad, f32, bf16):
    """All in one 256-row tile, two of keys; some in a wave's 32 rows together."""
    check(hq, hkv, d, SHORT, bad, f32=f32, bf16=bf16, poison=ALL)


def test_many_short_sequences():
    """More work-groups than run at once: tiles of 256 rows."""
    for bad in (0, 151, 152, 299):
        check(32, 8, 128, [100, 7, 30] * 100, bad, bf16=True)


@pytest.mark.parametrize("d", (64, 128))
def test_short_beside_long(d):
    """A long sequence's work-groups in the same launch, 128 rows each (two key groups)."""
    for bad in (0, 1, 3, 4):
        check(4, 2, d, [700, 30, 31, 90, 120], bad)


@pytest.mark.parametrize("d", (64, 128))
def test_short_neighbours_with_blocks(d):
    """By blocks, with token-causal segments."""
    lens = [40, 25, 60, 3, 70]
    blocks = [0, 10, 40, 65, 65, 90, 125, 128, 160, 198]
    text = [5, 30, 41, 65, 90, 100, 125, 150, 160]
    for bad in range(5):
        check(4, 2, d, lens, bad, blocks=blocks)
        check(4, 2, d, lens, bad, blocks=blocks, text=text)


@pytest.mark.parametrize("lens,bad", (([260] * 107, 50), ([260] * 171, 80), ([20500, 20500], 0), ([20500, 20500], 1), ([700] * 58, 29)))
def test_past_the_tables_of_the_gradients(lens, bad):
    """More key or row items than a launch's table holds: tiles of any neighbours."""
    check(2, 1, 64, lens, bad, bf16=True)


@pytest.mark.parametrize("lens,bad", (([300] * 450, 211), ([7] * 20000, 9000), ([3, 500] * 300, 301)))
def test_past_the_tables_of_the_forward(lens, bad):
    check(1, 1, 128, lens, bad)
    check(2, 2, 64, lens, bad, f32=True)


def test_a_sequence_all_bad():
    """Every value of a sequence, and of several, in all inputs at once."""
    gs.say("[gpu] packed, whole sequences not finite")
    hq, hkv, d = 4, 2, 64
    seqs = np.concatenate(([0], np.cumsum(SHORT)))
    T = int(seqs[-1])
    x = [rnd(1, T, hq, d), rnd(2, T, hkv, d), rnd(3, T, hkv, d), rnd(4, T, hq, d)]
    clean = calls(*x, pair(seqs), None, None, False, False)
    gone = [1, 3, 8]
    rows = torch.cat([torch.arange(int(seqs[s]), int(seqs[s + 1])) for s in gone]).to(DEV)
    rest = torch.tensor([i for i in range(T) if not any(seqs[s] <= i < seqs[s + 1] for s in gone)], device=DEV)
    for t in x:
        t[rows] = NAN
    got = calls(*x, pair(seqs), None, None, False, False)
    for p, c in zip(got, clean):
        assert torch.equal(p[rest], c[rest]) and not p[rows].isfinite().any()


@pytest.mark.parametrize("d", (64, 128))
def test_views(d):
    """Heads of one fused projection, outputs and gradients into views, tokens behind the
    last sequence, captured into a graph and replayed on other values."""
    gs.say(f"[gpu] packed, views, x {d}")
    hq, hkv, tail = 4, 2, 9
    lens = [*SHORT, 300]
    seqs = pair(np.concatenate(([0], np.cumsum(lens))))
    T = int(seqs[0][-1])
    fused, do = rnd(1, T + tail, hq + 2 * hkv, d), rnd(2, T + tail, hq, d)
    fused[T:], do[T:] = NAN, NAN
    first = fused.clone()
    q, k, v = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
    wide = torch.full((T + tail, 2 * hq, d), 7.0, dtype=torch.bfloat16, device=DEV)
    dfused = torch.full((T + tail, hq + 2 * hkv, d), 7.0, device=DEV)
    lse = torch.full((hq, T + tail), 7.0, device=DEV)
    space = torch.empty(ws.prefill_packed_bwd_workspace_bytes(T + tail, hq, hkv), dtype=torch.uint8, device=DEV)

    def run():
        ws.block_causal_prefill_packed(q, k, v, seqs, out=wide[:, 1::2], lse=lse)
        ws.block_causal_prefill_packed_bwd(q, k, v, wide[:, 1::2], do, lse, seqs, dq=dfused[:, :hq], dk=dfused[:, hq:hq + hkv],
                                           dv=dfused[:, hq + hkv:], workspace=space)

    run()
    clean = [t.clone() for t in (wide, dfused, lse)]
    assert all(t.isfinite().all() for t in clean) and (wide[:, ::2] == 7).all() and (wide[T:] == 7).all() and (dfused[T:] == 7).all()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
        run()
    torch.cuda.synchronize()
    for bad in (1, 4, 8, 9, None):
        fused.copy_(first)
        rest = torch.ones(T + tail, dtype=torch.bool, device=DEV)
        if bad is not None:
            a, e = seqs[0][bad:bad + 2].tolist()
            fused[(a + e) // 2, :, 5] = INF
            rest[a:e] = False
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip((wide, dfused, lse.T), (clean[0], clean[1], clean[2].T)):
            assert torch.equal(got[rest], want[rest]), bad
            assert bad is None or not got[~rest].isfinite().all()
