"""The windowed and 4-bit operators as a session uses them together: streaming
with a bounded set of recycled pages against the whole-sequence call, training
through it, decode and units over a 4-bit history, HIP-graph replays, other
streams, both marshallings."""
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


def _units(seed, n):
    """Lengths and text tokens of n units; now and then a decode step."""
    g = np.random.default_rng(seed)
    lens = [int(x) for x in g.choice([1, 2, 40, 90, 130], size=n)]
    return lens, [n if n <= 2 else int(g.integers(0, 6)) for n in lens]


def test_windowed_session_in_a_few_recycled_pages():
    """One session streamed unit by unit, each committed by its own step, in a
    pool that holds the sinks, the window and one unit: pages that leave the
    window are given back and used again.  Every unit's output is what the
    windowed prefill of the whole session says, and so are its gradients'
    operands."""
    Hq, Hkv, D, window, sinks = 8, 2, 128, 300, 70
    lens, text = _units(3, 24)
    off = np.concatenate(([0], np.cumsum(lens)))
    starts = off[1:] - text
    L = int(off[-1])
    q, k, v, do = _randn(1, 1, L, Hq, D), _randn(2, 1, L, Hkv, D), _randn(3, 1, L, Hkv, D), _randn(4, 1, L, Hq, D)
    lo, hi = ref.ranges(off, starts, window)
    want = ref.attend(q[0], k[0], v[0], lo, hi, sinks, D ** -0.5, dout=do[0])
    per = -(-L // 64)
    pages = 2 + -(-window // 64) + 1 + -(-max(lens) // 64) + 1
    assert pages < per - 3   # the session does not fit
    cache = ws.PagedCache.allocate(pages, Hkv, D, torch.full((1, per), -1), device=DEV, fill_bits=0x7FC1)
    free, table = list(range(pages)), np.full(per, -1)
    for n, (s, e) in enumerate(zip(off[:-1], off[1:])):
        s, e = int(s), int(e)
        for p in range(per):   # pages behind the sinks that no row can see any more
            if table[p] >= 0 and 64 * p >= sinks and 64 * (p + 1) <= s - window:
                cache.k_pool[table[p]] = float("nan")
                cache.v_pool[table[p]] = float("nan")
                free.append(int(table[p]))
                table[p] = -1
        for p in range(s // 64, -(-e // 64)):
            if table[p] < 0:
                table[p] = free.pop(0)
        step = ws.PagedCache(cache.k_pool, cache.v_pool, torch.from_numpy(table[None].copy()))
        out, lse = ws.block_causal_attn_fwd(q[:, s:e], k[:, s:e], v[:, s:e], step, _pair([s]), fuse_append=True,
                                            want_lse=True, text_starts=_pair([e - s - text[n]]), window=window, sinks=sinks)
        torch.cuda.synchronize()
        ref.check(f"unit {n}", out[0], tuple(x[s:e] for x in want["out"]))
        ref.check(f"unit {n} lse", lse[0], tuple(x[:, s:e] for x in want["lse"]))
    win = dict(text_starts=_pair(starts[None]), window=window, sinks=sinks)
    out, lse = ws.block_causal_prefill(q, k, v, _pair(off[None]), want_lse=True, **win)
    ref.check("prefill", out[0], want["out"])
    grads = ws.block_causal_prefill_bwd(q, k, v, out, do, lse, _pair(off[None]), grad_dtype=torch.bfloat16, **win)
    torch.cuda.synchronize()
    for name, x in zip(("dq", "dk", "dv"), grads):
        ref.check(name, x[0], want[name], bf16=True)


def test_a_window_past_the_history_is_no_window():
    """The windowed calls with a window that reaches the first token agree with
    the calls without one (to the difference of their roundings)."""
    B, L, Hq, Hkv, D = 2, 700, 6, 2, 64
    q, k, v = _randn(1, B, L, Hq, D), _randn(2, B, L, Hkv, D), _randn(3, B, L, Hkv, D)
    off = _pair([[0, 100, 100, 650, 700]] * B)
    a, la = ws.block_causal_prefill(q, k, v, off, want_lse=True)
    b, lb = ws.block_causal_prefill(q, k, v, off, want_lse=True, window=L)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(la, lb)   # the same arithmetic tile by tile


def test_4bit_session_of_units_and_decode_steps():
    """A session over a 4-bit history: units and decode steps in turn (both
    kernels), each committed by its own step, each against float64 over the
    rounded history; at the end the cache holds every token, rounded once."""
    B, Hq, Hkv, D = 2, 16, 4, 64
    lens, text = _units(5, 14)
    off = np.concatenate(([0], np.cumsum(lens)))
    L, first = int(off[-1]), [1000, 0]
    total = [f + L for f in first]
    per = -(-max(total) // 64)
    order = torch.randperm(B * per, generator=torch.Generator().manual_seed(1)).reshape(B, per)
    cache = ws.PagedCache4.allocate(B * per, Hkv, D, order, device=DEV)
    cache.pool.fill_(255)
    k, v = ([_randn(seed + b, max(total), Hkv, D) for b in range(B)] for seed in (10, 20))
    q = _randn(30, B, L, Hq, D)
    ws.kv_append(cache, _pair([0, 0]), torch.stack([x[:1000] for x in k]), torch.stack([x[:1000] for x in v]),
                 new_lens=_pair(first))
    rk, rv = [cache4_ref.rounded(x) for x in k], [cache4_ref.rounded(x) for x in v]
    kinds = set()
    for n, (s, e) in enumerate(zip(off[:-1], off[1:])):
        s, e = int(s), int(e)
        kinds.add((e - s) * Hq // Hkv <= 32)
        at = [f + s for f in first]
        kn, vn = (torch.stack([x[b][at[b]:at[b] + e - s] for b in range(B)]) for x in (k, v))
        out, lse = ws.block_causal_attn_fwd(q[:, s:e], kn, vn, cache, _pair(at), fuse_append=True, want_lse=True,
                                            text_starts=_pair([e - s - text[n]] * B))
        torch.cuda.synchronize()
        for b in range(B):
            lo, hi = ref.step_ranges(at[b], e - s, e - s - text[n], 2 ** 31)
            want = ref.attend(q[b, s:e], torch.cat((rk[b][:at[b]], kn[b])), torch.cat((rv[b][:at[b]], vn[b])), lo, hi, 0,
                              D ** -0.5)
            ref.check(f"unit {n} stream {b}", out[b], want["out"])
            ref.check(f"unit {n} stream {b} lse", lse[b], want["lse"])
    assert kinds == {True, False}
    for b in range(B):
        gk, gv = ws.kv_read(ws.PagedCache4(cache.pool, cache.page_table_host[b:b + 1]), _pair([0]), total[b])
        assert torch.equal(gk[0], rk[b][:total[b]]) and torch.equal(gv[0], rv[b][:total[b]])


def _calls(four):
    """Calls of every new entry point over fixed buffers, and their outputs."""
    Hq, Hkv, D, caches = 8, 2, 128, [1500, 333]
    lens = _pair(caches)
    per = -(-(max(caches) + 200) // 64)
    table = torch.randperm(2 * per, generator=torch.Generator().manual_seed(2)).reshape(2, per)
    if four:
        cache = ws.PagedCache4.allocate(2 * per, Hkv, D, table, device=DEV)
        cache.pool.fill_(255)
    else:
        cache = ws.PagedCache.allocate(2 * per, Hkv, D, table, device=DEV, fill_bits=0x7FC1)
    ws.kv_append(cache, _pair([0, 0]), _randn(1, 2, 1500, Hkv, D), _randn(2, 2, 1500, Hkv, D), new_lens=lens)
    res, calls = {}, []
    for Lq in (3, 4, 150):
        q, k, v = _randn(Lq, 2, Lq, Hq, D), _randn(Lq + 1, 2, Lq, Hkv, D), _randn(Lq + 2, 2, Lq, Hkv, D)
        out, lse = torch.empty_like(q), torch.empty(2, Hq, Lq, device=DEV)
        win = {} if four else dict(window=700, sinks=65)
        res[f"out{Lq}"], res[f"lse{Lq}"] = out, lse
        calls.append(lambda q=q, k=k, v=v, out=out, lse=lse, win=win, Lq=Lq: ws.block_causal_attn_fwd(
            q, k, v, cache, lens, fuse_append=Lq == 150, out=out, lse=lse, **win))
    if four:
        res["pool"] = cache.pool
        rk, rv = torch.empty(2, 160, Hkv, D, dtype=torch.bfloat16, device=DEV), torch.empty(2, 160, Hkv, D, dtype=torch.bfloat16, device=DEV)
        k2 = _randn(9, 2, 10, Hkv, D)
        at, start = _pair([1650, 483]), _pair(caches)
        res["k"], res["v"] = rk, rv
        calls.append(lambda: ws.kv_append(cache, at, k2, k2))
        calls.append(lambda: ws.kv_read(cache, start, 160, k=rk, v=rv))
        return res, calls
    res["kp"], res["vp"] = cache.k_pool, cache.v_pool
    L = 900
    q, k, v, do = _randn(11, 1, L, Hq, D), _randn(12, 1, L, Hkv, D), _randn(13, 1, L, Hkv, D), _randn(14, 1, L, Hq, D)
    off = _pair([[0, 200, 450, L]])
    out, lse = torch.empty_like(q), torch.empty(1, Hq, L, device=DEV)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    win = dict(window=150, sinks=10)
    res.update(out=out, lse=lse, dq=dq, dk=dk, dv=dv)
    calls.append(lambda: ws.block_causal_prefill(q, k, v, off, out=out, lse=lse, **win))
    calls.append(lambda: ws.block_causal_prefill_bwd(q, k, v, out, do, lse, off, dq=dq, dk=dk, dv=dv, **win))
    return res, calls


@pytest.mark.parametrize("four", (False, True))
def test_graph_replays_match_eager(four):
    """All calls captured into one graph; three replays, with eager work and
    synchronisation in between, give the eager results bit for bit."""
    gs.say(f"[gpu] graph of the new calls, four={four}")
    res, calls = _calls(four)
    for c in calls:
        c()
    torch.cuda.synchronize()
    want = {n: t.clone() for n, t in res.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for c in calls:
            c()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for c in calls:
            c()
    other, more = _calls(not four)
    for rep in range(3):
        gs.say(f"[gpu] replay {rep}")
        for n, t in res.items():
            if "pool" not in n and n not in ("kp", "vp"):
                t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        for c in more:   # eager work between replays, other workspaces
            c()
        torch.cuda.synchronize()
        for n, t in res.items():
            assert torch.equal(t.view(torch.uint8), want[n].view(torch.uint8)), (rep, n)


@pytest.mark.parametrize("four", (False, True))
def test_two_streams_at_once(four):
    """The same calls from two side streams at once, each with its own buffers,
    behind work that delays one of them: the results of one stream alone."""
    gs.say(f"[gpu] the new calls from two streams, four={four}")
    res, calls = _calls(four)
    for c in calls:
        c()
    torch.cuda.synchronize()
    want = {n: t.clone() for n, t in res.items()}
    pair = [_calls(four), _calls(four)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    slow = torch.randn(4096, 4096, device=DEV)
    with torch.cuda.stream(streams[0]):
        for _ in range(4):
            slow = slow @ slow * 1e-4
    for i in range(len(calls)):
        for s, (_, cs) in zip(streams, pair):
            with torch.cuda.stream(s):
                cs[i]()
    torch.cuda.synchronize()
    for got, _ in pair:
        for n, t in got.items():
            assert torch.equal(t.view(torch.uint8), want[n].view(torch.uint8)), n


class _Declines:
    """Takes no call, so every call goes through the Python code."""

    def __getattr__(self, name):
        return lambda *_: None


def _outcome(f):
    try:
        r = f()
        torch.cuda.synchronize()
    except Exception as e:   # compared below
        return type(e).__name__, str(e)
    return [t.clone() for t in (r if isinstance(r, (tuple, list)) else (r,)) if t is not None]


def test_both_marshallings_agree(monkeypatch):
    """Native and ctypes marshalling: the same bits, the same refusals."""
    Hq, Hkv, D = 4, 2, 64
    q, k, v = _randn(1, 2, 5, Hq, D), _randn(2, 2, 5, Hkv, D), _randn(3, 2, 5, Hkv, D)
    table = torch.arange(8).reshape(2, 4)
    full = ws.PagedCache.allocate(8, Hkv, D, table, device=DEV, fill_bits=0)
    four = ws.PagedCache4.allocate(8, Hkv, D, table, device=DEV)
    four.pool.zero_()
    off, lens = _pair([[0, 2, 5]] * 2), _pair([70, 5])
    o, lse = ws.block_causal_prefill(q, k, v, off, want_lse=True, window=1)
    calls = [
        lambda: ws.block_causal_attn_fwd(q, k, v, full, lens, window=3, sinks=2, want_lse=True),
        lambda: ws.block_causal_attn_fwd(q, k, v, full, lens, window=3, out_dtype=torch.float32, new_lens=_pair([5, 2])),
        lambda: ws.block_causal_attn_fwd(q, k, v, full, [70, 5], window=3, text_starts=[1, 5]),
        lambda: ws.block_causal_attn_fwd(q, k, v, full, _pair([300, 5]), window=300),        # capacity
        lambda: ws.block_causal_attn_fwd(q, k[:, :4], v, full, lens, window=3),              # shape
        lambda: ws.block_causal_attn_fwd(q, k, v, full, lens, window=3, workspace=torch.empty(0, device=DEV)),
        lambda: ws.block_causal_prefill(q, k, v, off, window=2, sinks=1, want_lse=True),
        lambda: ws.block_causal_prefill(q, k, v, _pair([[0, 2, 4]] * 2), window=2),          # offsets
        lambda: ws.block_causal_prefill(q, None, None, off, cache=full, window=2),
        lambda: ws.block_causal_prefill_bwd(q, k, v, o, o, lse, off, window=1),
        lambda: ws.block_causal_prefill_bwd(q, k, v, o, o, lse, off, window=1, grad_dtype=torch.bfloat16),
        lambda: ws.block_causal_prefill_bwd(q, k, v, o, o, lse, off, window=1, dq=torch.empty_like(q)),   # mixed
        lambda: ws.block_causal_attn_fwd(q, k, v, four, lens, want_lse=True),
        lambda: ws.block_causal_attn_fwd(q, k, v, four, [70, 5], fuse_append=True),
        lambda: ws.block_causal_attn_fwd(q, k, v, four, lens, text_starts=_pair([0, 9])),    # offsets
        lambda: ws.block_causal_attn_fwd(q.repeat(1, 1, 1, 2), k, v, four, lens),            # head_dim
        lambda: (ws.kv_append(four, lens, k, v), four.pool)[1],
        lambda: (ws.kv_append(four, [70, 5], k, v, new_lens=[5, 0]), four.pool)[1],
        lambda: ws.kv_append(four, _pair([252, 5]), k, v),                                   # capacity
        lambda: ws.kv_read(four, lens, 5),
        lambda: ws.kv_read(four, [70, 5], 5, k=torch.empty_like(k)),
        lambda: ws.kv_read(four, lens, 5, k=torch.empty_like(q)),                            # shape
        lambda: ws.kv_read(four, lens, 0),
        lambda: ws.kv_read(four, _pair([70, 5, 6]), 5),                                      # table rows
        lambda: ws.kv_append(four, lens, k[:, :0], v[:, :0]),
    ]
    for i, call in enumerate(calls):
        native = _outcome(call)
        with monkeypatch.context() as m:
            m.setattr(ws, "_NATIVE", _Declines())
            python = _outcome(call)
        if isinstance(native, tuple):
            assert native == python, i
        else:
            assert len(native) == len(python), i
            for a, b in zip(native, python):
                assert a.dtype == b.dtype and torch.equal(a.view(torch.uint8), b.view(torch.uint8)), i


@pytest.mark.parametrize("Lq", (3, 40))
def test_a_nan_reaches_the_rows_that_see_it_and_no_other(Lq):
    """A committed block with a NaN (and one with an infinity) in a 4-bit cache:
    the heads that read it give NaN, the other heads and streams do not."""
    Hq, Hkv, D = 4, 2, 128
    cache = ws.PagedCache4.allocate(8, Hkv, D, torch.arange(8).reshape(2, 4), device=DEV)
    cache.pool.fill_(255)
    k, v = _randn(1, 2, 100, Hkv, D), _randn(2, 2, 100, Hkv, D)
    k[0, 17, 1, 40], v[1, 99, 0, 3] = float("nan"), float("inf")
    ws.kv_append(cache, _pair([0, 0]), k, v)
    q, kn = _randn(3, 2, Lq, Hq, D), _randn(4, 2, Lq, Hkv, D)
    for dtype in (torch.bfloat16, torch.float32):
        out = ws.block_causal_attn_fwd(q, kn, kn, cache, _pair([100, 100]), out_dtype=dtype)
        torch.cuda.synchronize()
        assert out[0, :, 2:].isnan().all() and not out[0, :, :2].isnan().any()
        assert out[1, :, :2, :32].isnan().all()   # the value's block of 32 head dims
        assert not out[1, :, 2:].isnan().any() and not out[1, :, :2, 32:].isnan().any()
    out = ws.block_causal_attn_fwd(q, kn, kn, cache, _pair([17, 99]))   # not reached
    assert not out.isnan().any()


def test_empty_calls():
    q, k = torch.empty(0, 4, 4, 64, dtype=torch.bfloat16, device=DEV), torch.empty(0, 4, 2, 64, dtype=torch.bfloat16, device=DEV)
    four = ws.PagedCache4.allocate(1, 2, 64, torch.zeros(1, 1), device=DEV)
    none = _pair(np.zeros(0))
    assert ws.block_causal_attn_fwd(q, k, k, four, none).shape == q.shape
    assert ws.kv_read(four, none, 3)[0].shape == (0, 3, 2, 64)
    assert ws.block_causal_prefill(q, k, k, _pair(np.zeros((0, 2))), window=3).shape == q.shape
    q1, k1 = torch.empty(1, 0, 4, 64, dtype=torch.bfloat16, device=DEV), torch.empty(1, 0, 2, 64, dtype=torch.bfloat16, device=DEV)
    assert ws.block_causal_attn_fwd(q1, k1, k1, four, _pair([0])).shape == q1.shape
    assert ws.block_causal_prefill(q1, k1, k1, _pair([[0, 0]]), window=0, sinks=0).shape == q1.shape
    dq, dk, dv = ws.block_causal_prefill_bwd(q1, k1, k1, q1, q1, torch.empty(1, 4, 0, device=DEV), _pair([[0, 0]]), window=2)
    assert dq.shape == q1.shape and dk.shape == k1.shape and dv.shape == k1.shape


@pytest.mark.parametrize("four", (False, True))
def test_refused_calls_change_nothing(four):
    """The last check of each call fails (the page of a committed token, the
    workspace): outputs, log-sum-exp, gradients and pools keep their bytes."""
    Hq, Hkv, D, Lq = 8, 2, 128, 40
    table = torch.tensor([[0, 1, 9]], dtype=torch.int32)   # 3 pages in the pool; page 9 is that of positions 128..
    if four:
        cache = ws.PagedCache4.allocate(3, Hkv, D, table, device=DEV)
        cache.pool.fill_(7)
        pools = [cache.pool]
    else:
        cache = ws.PagedCache.allocate(3, Hkv, D, table, device=DEV, fill_bits=0x4040)
        pools = [cache.k_pool, cache.v_pool]
    q, k, v = _randn(1, 1, Lq, Hq, D), _randn(2, 1, Lq, Hkv, D), _randn(3, 1, Lq, Hkv, D)
    out, lse = torch.full_like(q, 7.0), torch.full((1, Hq, Lq), 3.0, device=DEV)
    grads = [torch.full_like(x, 5.0) for x in (q, k, v)]
    kept = [out, lse, *grads, *pools]
    before = [t.clone() for t in kept]
    win = {} if four else dict(window=50, sinks=3)
    off, small = _pair([[0, Lq]]), torch.empty(64, dtype=torch.uint8, device=DEV)
    calls = {"WS_ERR_PAGE": lambda: ws.block_causal_attn_fwd(q, k, v, cache, _pair([100]), fuse_append=True, out=out, lse=lse, **win)}
    if four:
        with pytest.raises(ws.WsError) as e:
            ws.kv_append(cache, _pair([100]), k, v)
        assert e.value.name == "WS_ERR_PAGE"
        with pytest.raises(ws.WsError) as e:
            ws.kv_read(cache, _pair([100]), Lq, k=grads[1], v=grads[2])
        assert e.value.name == "WS_ERR_PAGE"
    else:
        calls["WS_ERR_WORKSPACE"] = lambda: ws.block_causal_prefill_bwd(
            q, k, v, q, q, lse, off, dq=grads[0], dk=grads[1], dv=grads[2], workspace=small, **win)
    for name, call in calls.items():
        with pytest.raises(ws.WsError) as e:
            call()
        assert e.value.name == name
    torch.cuda.synchronize()
    for t, was in zip(kept, before):
        assert torch.equal(t.view(torch.uint8), was.view(torch.uint8))
