"""Packed attention and linear attention as a model uses them, on the GPU: layers
of both over one packed batch with their gradients, prompts and the steps behind
them, captured into a graph, on two streams, in views, far apart in memory.
Each stage is checked against its definition in 64 bits on the very tensors that
it was given (tests/window_ref.py, tests/linear_ref.py state the bounds)."""
import numpy as np
import pytest
import torch

import paper_2606_25041_amd as ws
from paper_2606_25041_amd import linear, packed
from tests import gpu_support as gs
from tests import linear_ref as lref
from tests import window_ref as ref
from tests.test_gpu_linear import check_bwd, close, decays, f64, offsets, pair, rnd, rnd32

pytestmark = pytest.mark.gpu
DEV = "cuda"
LENS = [70, 1, 0, 300, 33, 128]


def check_attn(q, k, v, lens, out, do=None, grads=(), bf16=True):
    a = 0
    for s, n in enumerate(lens):
        e = a + n
        lo, hi = np.zeros(n, np.int64), np.arange(1, n + 1)
        if n:
            want = ref.attend(q[a:e], k[a:e], v[a:e], lo, hi, 0, q.shape[2] ** -0.5, dout=None if do is None else do[a:e])
            ref.check(f"out {s}", out[a:e], want["out"])
            for name, x in zip(("dq", "dk", "dv"), grads):
                ref.check(f"{name} {s}", x[a:e], want[name], bf16=bf16)
        a = e


def check_linear(q, k, v, ld, lens, out, before=None, after=None, dt=torch.bfloat16):
    scale, a = q.shape[2] ** -0.5, 0
    for s, n in enumerate(lens):
        e = a + n
        zero = np.zeros((k.shape[1], q.shape[2], q.shape[2]))
        want, S, mags, A = lref.forward(f64(q[a:e]), f64(k[a:e]), f64(v[a:e]), f64(ld), zero if before is None else before[s])
        close(f"linear out {s}", out[a:e], want * scale, lref.out_bound(want, mags, n, dt, scale))
        if after is not None:
            close(f"state {s}", after[s], S, lref.state_bound(A, n))
        a = e


def check_linear_bwd(q, k, v, do, ld, lens, grads):
    scale, a = q.shape[2] ** -0.5, 0
    zero = np.zeros((k.shape[1], q.shape[2], q.shape[2]))
    G = q.shape[1] // k.shape[1]
    for s, n in enumerate(lens):
        e = a + n
        want = lref.gradients(f64(q[a:e]), f64(k[a:e]), f64(v[a:e]), f64(do[a:e]), f64(ld), zero, zero, scale)
        for name, x in zip(("dq", "dk", "dv"), grads):
            w, mags = want[name]
            close(f"linear {name} {s}", x[a:e], w * scale, lref.out_bound(w, mags, n * G, torch.bfloat16, scale))
        a = e


@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (4, 4, 128)])
def test_layers_and_their_gradients(hq, hkv, d):
    """A softmax layer whose outputs are the next, linear, layer's queries."""
    gs.say(f"[gpu] softmax layer, then linear layer, {hq}/{hkv} x {d}")
    T, seqs = sum(LENS), offsets(LENS)
    q, k, v, do = rnd(1, T, hq, d), rnd(2, T, hkv, d), rnd(3, T, hkv, d), rnd(4, T, hq, d)
    k2, v2, ld = rnd(5, T, hkv, d), rnd(6, T, hkv, d), decays(hkv)
    mid, lse = ws.block_causal_prefill_packed(q, k, v, seqs, want_lse=True)
    out = ws.linear_attn_prefill(mid, k2, v2, ld, seqs)
    dmid, dk2, dv2 = ws.linear_attn_prefill_bwd(mid, k2, v2, do, ld, seqs)[:3]
    grads = ws.block_causal_prefill_packed_bwd(q, k, v, mid, dmid, lse, seqs, grad_dtype=torch.bfloat16)
    torch.cuda.synchronize()
    check_attn(q, k, v, LENS, mid, dmid, grads)
    check_linear(mid, k2, v2, ld, LENS, out)
    check_linear_bwd(mid, k2, v2, do, ld, LENS, (dmid, dk2, dv2))


def test_prompts_and_the_steps_behind_them():
    """Prompts of different lengths in one batch through both kinds of layer, their
    keys to a paged cache and their states to a pool; then three tokens of every
    session against both, one at a time."""
    hq, hkv, d, lens, new = 8, 2, 128, [70, 1, 130, 64], 3
    gs.say(f"[gpu] prompts {lens} and {new} steps, {hq}/{hkv} x {d}")
    B, T, seqs = len(lens), sum(lens), offsets(lens)
    q, k, v = rnd(1, T, hq, d), rnd(2, T, hkv, d), rnd(3, T, hkv, d)
    qs, ks, vs = rnd(4, B, new, hq, d), rnd(5, B, new, hkv, d), rnd(6, B, new, hkv, d)
    ld = decays(hkv)
    cache = ws.PagedCache.allocate(4 * B, hkv, d, torch.arange(4 * B).view(B, 4), fill_bits=gs.NAN_BITS)
    state = ws.LinearState.allocate(B + 1, hkv, d, pair([2, 4, 0, 1]))
    out = ws.block_causal_prefill_packed(q, k, v, seqs)
    lout = ws.linear_attn_prefill(q, k, v, ld, seqs, state=state, reset=True)
    at = np.concatenate(([0], np.cumsum(lens)))
    for b in range(B):   # the packed keys are the cache's first tokens
        one = ws.PagedCache(cache.k_pool, cache.v_pool, torch.arange(4 * b, 4 * b + 4).view(1, 4))
        ws.kv_append(one, [0], k[None, at[b]:at[b + 1]], v[None, at[b]:at[b + 1]])
    steps, lsteps = [], []
    for t in range(new):
        one = [x[:, t:t + 1] for x in (qs, ks, vs)]
        steps.append(ws.block_causal_attn_fwd(*one, cache, [n + t for n in lens], fuse_append=True))
        lsteps.append(ws.linear_attn_step(*one, ld, state))
    torch.cuda.synchronize()
    check_attn(q, k, v, lens, out)
    check_linear(q, k, v, ld, lens, lout)
    scale = d ** -0.5
    for b in range(B):
        n = lens[b]
        K, V = torch.cat((k[at[b]:at[b + 1]], ks[b])), torch.cat((v[at[b]:at[b + 1]], vs[b]))
        lo, hi = np.zeros(new, np.int64), n + 1 + np.arange(new)
        want = ref.attend(qs[b], K, V, lo, hi, 0, scale)
        ref.check(f"step of {b}", torch.cat(steps, 1)[b], want["out"])
        # the recurrence over all of the session; the steps' own bound, and what the
        # prompt's state brings with it (state_bound, through the query)
        allq = torch.cat((q[at[b]:at[b + 1]], qs[b]))
        w, S, mags, A = lref.forward(f64(allq), f64(K), f64(V), f64(ld), np.zeros((hkv, d, d)))
        bound = lref.step_bound(w[n:], mags[2][n:], new, torch.bfloat16, scale) + \
            (2.0 ** -20 + (8 * lref.chunks(n) + 64) * 2.0 ** -24) * mags[2][n:] * scale
        close(f"linear step of {b}", torch.cat(lsteps, 1)[b], w[n:] * scale, bound)
        close(f"state of {b}", state.pool[[2, 4, 0, 1][b]], S, lref.state_bound(A, n) + (3 * new + 8) * 2.0 ** -24 * A)
    assert (state.pool[3] == 0).all()


def run_all(x, ld, seqs, space, lspace, pool, start, step, slots):
    """A batch through every operator here; in place on the pool."""
    q, k, v, do = x
    pool.copy_(start)
    state = ws.LinearState(pool, slots)
    out, lse = ws.block_causal_prefill_packed(q, k, v, seqs, want_lse=True)
    grads = ws.block_causal_prefill_packed_bwd(q, k, v, out, do, lse, seqs, workspace=space)
    lgrads = ws.linear_attn_prefill_bwd(q, k, v, do, ld, seqs, state=state, workspace=lspace)
    lout = ws.linear_attn_prefill(q, k, v, ld, seqs, state=state, workspace=lspace)
    sout = ws.linear_attn_step(*step, ld, state)
    return [out, lse, *grads, *[g for g in lgrads if g is not None], lout, sout, pool]


def workload(seed, hq=4, hkv=2, d=64):
    T, S = sum(LENS), len(LENS)
    x = rnd(seed, T, hq, d), rnd(seed + 1, T, hkv, d), rnd(seed + 2, T, hkv, d), rnd(seed + 3, T, hq, d)
    step = rnd(seed + 4, S, 1, hq, d), rnd(seed + 5, S, 1, hkv, d), rnd(seed + 6, S, 1, hkv, d)
    space = torch.empty(ws.prefill_packed_bwd_workspace_bytes(T, hq, hkv), dtype=torch.uint8, device=DEV)
    lspace = torch.empty(ws.linear_workspace_bytes(S, T, hq, hkv, d), dtype=torch.uint8, device=DEV)
    start = rnd32(seed + 7, S, hkv, d, d)
    return x, decays(hkv), offsets(LENS), space, lspace, torch.empty_like(start), start, step, pair(list(range(S)))


def test_captured_and_replayed():
    """Replays between eager work on the same workspaces, new inputs each time."""
    gs.say("[gpu] all operators in a graph, replayed")
    work = workload(20)
    run_all(*work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run_all(*work)
    for turn in range(4):
        for old, new in zip(work[0], workload(100 * turn + 7)[0]):
            old.copy_(new)
        want = [t.clone() for t in run_all(*work)]
        torch.cuda.synchronize()
        for t in held:
            t.fill_(3)
        work[3].fill_(0xFF), work[4].fill_(0xFF)   # (workspaces hold nothing between calls)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), turn
        _ = sum(float(t.float().sum()) for t in want)


def test_two_streams():
    """Two batches at once, each on a stream of its own with its own workspaces."""
    gs.say("[gpu] all operators on two streams")
    works = [workload(30), workload(60, hq=8, hkv=8, d=128)]
    want = [[t.clone() for t in run_all(*w)] for w in works]
    streams = [torch.cuda.Stream() for _ in works]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for s, w in zip(streams, works):
            with torch.cuda.stream(s):
                got.append(run_all(*w))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(g, w))


def test_views():
    """Rows of a fused projection in, a part of a wider tensor out; what lies
    between and behind the last sequence stays as it was, and may be anything."""
    hq, hkv, d, lens = 4, 2, 64, [40, 0, 91]
    gs.say("[gpu] views of packed tensors")
    T, tail, seqs = sum(lens), 9, offsets(lens)
    fused = rnd(1, T + tail, (hq + 2 * hkv) * d)
    fused[T:] = float("nan")
    q, k, v = (fused[:, a * d:(a + h) * d].view(T + tail, h, d) for a, h in ((0, hq), (hq, hkv), (hq + hkv, hkv)))
    do = rnd(2, hq, T + tail, d).transpose(0, 1)
    ld = decays(hkv)
    wide = lambda h: torch.full((T + tail, h + 1, d + 8), 7.0, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    part = lambda x: x[:, 1:, :d]  # noqa: E731
    o, lo = wide(hq), wide(hq)
    g, lg = [wide(h) for h in (hq, hkv, hkv)], [wide(h) for h in (hq, hkv, hkv)]
    _, lse = ws.block_causal_prefill_packed(q, k, v, seqs, out=part(o), want_lse=True)
    ws.block_causal_prefill_packed_bwd(q, k, v, part(o), do, lse, seqs, dq=part(g[0]), dk=part(g[1]), dv=part(g[2]))
    ws.linear_attn_prefill(q, k, v, ld, seqs, out=part(lo))
    ws.linear_attn_prefill_bwd(q, k, v, do, ld, seqs, dq=part(lg[0]), dk=part(lg[1]), dv=part(lg[2]))
    torch.cuda.synchronize()
    check_attn(q, k, v, lens, part(o), do, [part(x) for x in g])
    check_linear(q, k, v, ld, lens, part(lo))
    check_linear_bwd(q, k, v, do, ld, lens, [part(x) for x in lg])
    for x in (o, lo, *g, *lg):
        part(x)[:T] = 7
        assert (x == 7).all()


def test_far_apart():
    """Tokens 16 MiB apart, states past 4 GiB: offsets of more than 32 bits."""
    hq, hkv, d, lens = 2, 1, 128, [100, 200]
    gs.say("[gpu] tokens and states far apart")
    T, seqs, st = sum(lens), offsets(lens), 2 ** 23 - 8
    room = torch.empty(T * st + 4 * hq * d, dtype=torch.bfloat16, device=DEV)
    views = [room.as_strided((T, h, d), (st, d, 1), a * d) for h, a in ((hq, 0), (hkv, 2), (hkv, 3), (hq, 4))]
    for x, s in zip(views, range(4)):
        x.copy_(rnd(s, *x.shape))
    q, k, v, do = views
    ld = decays(hkv)
    out, lse = ws.block_causal_prefill_packed(q, k, v, seqs, want_lse=True)
    grads = ws.block_causal_prefill_packed_bwd(q, k, v, out, do, lse, seqs, grad_dtype=torch.bfloat16)
    check_attn(q, k, v, lens, out, do, grads)
    slots = 70000
    pool = torch.empty(slots, hkv, d, d, device=DEV)
    at = [slots - 1, 66000]
    pool[at] = rnd32(9, 2, hkv, d, d)
    before = f64(pool[at])
    lout = ws.linear_attn_prefill(q, k, v, ld, seqs, state=ws.LinearState(pool, pair(at)))
    check_linear(q, k, v, ld, lens, lout, before, pool[at])
    check_linear_bwd(q, k, v, do, ld, lens, ws.linear_attn_prefill_bwd(q, k, v, do, ld, seqs)[:3])
    step = rnd(11, 2, 1, hq, d), rnd(12, 2, 1, hkv, d), rnd(13, 2, 1, hkv, d)
    small = pool[at].clone()
    a = ws.linear_attn_step(*step, ld, ws.LinearState(pool, pair(at)))
    b = ws.linear_attn_step(*step, ld, ws.LinearState(small, pair([0, 1])))
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(pool[at], small)


@pytest.mark.parametrize("f32", (False, True))
@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 64), (3, 1, 128)])
@pytest.mark.parametrize("lens", ([17000, 1, 130], [700, 40]))
def test_more_tokens_than_run_at_once(lens, hq, hkv, d, f32):
    """Several query heads in a work-group, and longer cells; and one each."""
    gs.say(f"[gpu] linear prefill {hq}/{hkv} x {d}, {lens}, f32={f32}")
    T, seqs = sum(lens), offsets(lens)
    q, k, v, ld = rnd(1, T, hq, d), rnd(2, T, hkv, d), rnd(3, T, hkv, d), decays(hkv)
    pool = rnd32(4, len(lens), hkv, d, d)
    before = f64(pool)
    dt = torch.float32 if f32 else torch.bfloat16
    out = ws.linear_attn_prefill(q, k, v, ld, seqs, state=ws.LinearState(pool, pair(list(range(len(lens))))), out_dtype=dt)
    check_linear(q, k, v, ld, lens, out, before, pool, dt)


def test_gradients_of_long_cells():
    gs.say("[gpu] linear gradients of 9000 tokens")
    check_bwd(3, 1, 64, [9000, 40], "spread", True)


@pytest.mark.parametrize("hkv,d,G", [(16, 128, 1), (8, 128, 3), (32, 64, 1)])
def test_steps_of_many_sequences(hkv, d, G):
    """Waves of 32 columns, as tests of few sequences take waves of 8; equal results
    of a sequence alone and among others up to the order of its sums."""
    B, n = 1024 * 32 // d // hkv + 3, 2
    gs.say(f"[gpu] linear step of {B} sequences, {hkv * G}/{hkv} x {d}")
    q, k, v, ld = rnd(1, B, n, hkv * G, d), rnd(2, B, n, hkv, d), rnd(3, B, n, hkv, d), decays(hkv)
    pool = rnd32(4, B, hkv, d, d)
    before = f64(pool)
    out = ws.linear_attn_step(q, k, v, ld, ws.LinearState(pool, pair(list(range(B)))), out_dtype=torch.float32)
    for b in (0, 1, B // 2, B - 1):
        want, S, mags, A = lref.forward(f64(q[b]), f64(k[b]), f64(v[b]), f64(ld), before[b])
        close(f"out of {b}", out[b], want * d ** -0.5, lref.step_bound(want, mags[2], n, torch.float32, d ** -0.5))
        close(f"state of {b}", pool[b], S, (3 * n + 8) * 2.0 ** -24 * A + 1e-37)


def test_a_slot_read_twice():
    """Uncommitted calls may read one state for several sequences; a call that
    commits may not."""
    gs.say("[gpu] one state for several sequences")
    pool, ld = rnd32(1, 2, 2, 64, 64), decays(2)
    q, k, v = rnd(2, 2, 4, 4, 64), rnd(3, 2, 4, 2, 64), rnd(4, 2, 4, 2, 64)
    twice, kept = ws.LinearState(pool, pair([1, 1])), pool.clone()
    both = ws.linear_attn_step(q, k, v, ld, twice, commit=False)
    for b in range(2):
        one = ws.linear_attn_step(q[b:b + 1], k[b:b + 1], v[b:b + 1], ld, ws.LinearState(pool, pair([1])), commit=False)
        assert torch.equal(one[0], both[b])
    seqs = offsets([4, 4])
    flat = lambda x: x.reshape(8, *x.shape[2:])  # noqa: E731
    out = ws.linear_attn_prefill(flat(q), flat(k), flat(v), ld, seqs, state=twice, commit=False)
    check_linear(flat(q), flat(k), flat(v), ld, [4, 4], out, f64(pool[[1, 1]]))
    assert torch.equal(pool, kept)
    for call in (lambda: ws.linear_attn_step(q, k, v, ld, twice),
                 lambda: ws.linear_attn_prefill(flat(q), flat(k), flat(v), ld, seqs, state=twice)):
        with pytest.raises(ws.WsError):
            call()
    torch.cuda.synchronize()
    assert torch.equal(pool, kept)


def test_both_ways_through_the_binding(monkeypatch):
    """The native module's calls and the ctypes ones: the same bits."""
    gs.say("[gpu] native and ctypes marshalling")
    work = workload(40)
    want = [t.clone() for t in run_all(*work)]

    class Declines:
        def __getattr__(self, name):
            return lambda *a: None

    for module in (linear, packed):
        monkeypatch.setattr(module, "_native", lambda: Declines())
    got = run_all(*work)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("n", (2, 3, 5))
def test_gradients_of_few_keys(n):
    """dQ and dK carry two roundings to bf16, that of dS and their own, each at most
    2^-8 of a value and, over values anywhere between two powers of two, at most
    2^-8 / sqrt(3) in the mean square: sqrt(2 / 3) 2^-8 of the norm together (D from
    a rounded output would add as much again where rows see few keys)."""
    hq, hkv, d, S = 2, 2, 64, 600
    gs.say(f"[gpu] packed gradients of {S} sequences of {n}")
    T, seqs = n * S, offsets([n] * S)
    q, k, v, do = (rnd(i, T, 2, d) for i in range(4))
    out, lse = ws.block_causal_prefill_packed(q, k, v, seqs, want_lse=True)
    dq, dk, _ = ws.block_causal_prefill_packed_bwd(q, k, v, out, do, lse, seqs, grad_dtype=torch.bfloat16)
    x = [t.cpu().double().view(S, n, hq, d).transpose(1, 2).contiguous() for t in (q, k, v, do)]
    s = x[0] @ x[1].transpose(2, 3).contiguous() * d ** -0.5
    p = s.masked_fill(~torch.ones(n, n, dtype=torch.bool).tril(), -torch.inf).softmax(3)
    dp = x[3] @ x[2].transpose(2, 3).contiguous()
    ds = p * (dp - (p * dp).sum(3, keepdim=True)) * d ** -0.5
    for name, got, want in (("dq", dq, ds @ x[1]), ("dk", dk, ds.transpose(2, 3).contiguous() @ x[0])):
        got = got.cpu().double().view(S, n, hq, d).transpose(1, 2)
        assert float((got - want).norm() / want.norm()) <= (2 / 3) ** 0.5 * 2.0 ** -8, name


@pytest.mark.parametrize("bad", (float("nan"), float("inf")))
def test_what_is_not_finite_stays_in_its_sequence(bad):
    """Linear attention: every other sequence's outputs, states and gradients bit for
    bit as without it, with sequences that share cells, chunks' tails and cell edges."""
    hq, hkv, d = 4, 2, 64
    lens, sick = [5, 90, 130, 1, 31, 260], (1, 4)
    gs.say(f"[gpu] {bad} in two of {len(lens)} sequences")
    T, S, seqs = sum(lens), len(lens), offsets(lens)
    at = np.concatenate(([0], np.cumsum(lens)))
    ld, start = decays(hkv), rnd32(9, S, hkv, d, d)

    def run(x, before):
        pool = before.clone()
        st = ws.LinearState(pool, pair(list(range(S))))
        q, k, v, do = x
        grads = ws.linear_attn_prefill_bwd(q, k, v, do, ld, seqs, state=st, dstate=before, want_dstate0=True)
        return ws.linear_attn_prefill(q, k, v, ld, seqs, state=st), pool, grads

    x = [rnd(1, T, hq, d), rnd(2, T, hkv, d), rnd(3, T, hkv, d), rnd(4, T, hq, d)]
    out, pool, grads = run(x, start)
    for t in x:
        for s in sick:
            t[at[s] + lens[s] // 2] = bad
    before = start.clone()
    before[4, 0, 3] = bad
    out2, pool2, grads2 = run(x, before)
    torch.cuda.synchronize()
    for s in range(S):
        if s not in sick:
            a, e = at[s], at[s + 1]
            assert torch.equal(out[a:e], out2[a:e]) and torch.equal(pool[s], pool2[s]), s
            assert all(torch.equal(g[a:e], h[a:e]) for g, h in zip(grads[:3], grads2[:3])), s
            assert torch.equal(grads[3][s], grads2[3][s]), s
    assert not torch.isfinite(out2[at[1]:at[2]].float()).all()
