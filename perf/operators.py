"""Operators that bound what a long session costs, and the calls that measure them.

Windowed attention: a streaming step, a whole-sequence prefill and the
gradients in which a token sees the first `sinks` tokens, the `window` tokens
before its block (a token-causal token: before itself) and its own block.  A
4-bit cache: committing tokens to it, reading them back, and the streaming
step over it.

For token i of the block [s, e) with segment start tau (tau = e: none):
    hi_i = max(tau, i + 1),   lo_i = (i if i >= tau else s) - window,
    key j is visible if j < hi_i and (j < sinks or j >= lo_i).
4-bit cache: 32 neighbouring head dims of a token and head share the scale 2^e,
e the least integer (in [-100, 125]) with amax <= 6 * 2^e; an element is x / 2^e
rounded to the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 (ties to the even code),
with its sign.  A step sees its own new block unrounded.

A case names its kind, its heads ("hq" x "hkv" x "d") and its sizes; lists of
lengths are texts.  Inputs come from the seed alone; lengths belong to the case.
"""
import math

import torch

own = False
PAGE = 64
DEV = "cuda"


def listed():
    return [
        # thinker decode: four sessions of different ages, one token each, over
        # the first page and the last 4096 tokens; expired pages are freed
        dict(name="window_decode", kind="wstep", hq=64, hkv=8, d=128, new=1, caches="131072,60011,9001,517",
             window=4096, sinks=64, text=True, fuse=True, f32=False, lse=False, new_lens=""),
        # four sessions ingest units of different lengths (text segments
        # token-causal), committed in the same launch
        dict(name="window_units_ragged", kind="wstep", hq=64, hkv=8, d=128, new=243,
             caches="131072,60011,24000,8190", window=16384, sinks=64, text=True, fuse=True, f32=False, lse=False,
             new_lens="145,110,163,243"),
        # performer: one 256-token block, a window that is no multiple of a
        # page, four sinks, the log-sum-exp kept
        dict(name="window_block", kind="wstep", hq=24, hkv=24, d=128, new=256, caches="22579", window=4001, sinks=4,
             text=False, fuse=False, f32=False, lse=True, new_lens=""),
        # a system prefill of 16 interleaved units from the paged cache
        dict(name="window_prefill_system", kind="wprefill", batch=1, hq=40, hkv=8, d=128, blocks=16, block=0, layout=4,
             window=777, sinks=17, paged=True, text=True, f32=False, lse=False),
        # two long histories, 64 blocks of 256
        dict(name="window_prefill_long", kind="wprefill", batch=2, hq=32, hkv=8, d=128, blocks=64, block=256,
             layout=0, window=4096, sinks=64, paged=False, text=False, f32=False, lse=False),
        # forward and gradients of an attention layer on 12 interleaved units
        dict(name="window_train_units", kind="wtrain", batch=1, hq=32, hkv=8, d=128, blocks=12, block=0, layout=9,
             window=500, sinks=5, text=True),
        # forward and gradients on two 16384-token sequences
        dict(name="window_train_long", kind="wtrain", batch=2, hq=32, hkv=8, d=128, blocks=64, block=256, layout=0,
             window=2048, sinks=64, text=False),
        # commit one average interleaved unit (174 tokens) at 4 bits and read
        # it back: the smallest call of the serving loop
        dict(name="cache4_append_unit", kind="append4", hq=64, hkv=8, d=128, new=174, caches="22579"),
        # two whole histories move into the 4-bit cache
        dict(name="cache4_append_history", kind="append4", hq=32, hkv=8, d=128, new=16384, caches="0,33"),
        # thinker decode over a 4-bit history: four sessions of different ages
        # each append 3 token-causal tokens, committed in the same launch
        dict(name="cache4_decode", kind="step4", hq=64, hkv=8, d=128, new=3, caches="131072,131007,60011,24000",
             text=True, fuse=True, f32=False, lse=False, new_lens=""),
        # six sessions of a small head_dim-64 model, odd block, f32 out and lse
        dict(name="cache4_step_d64_f32", kind="step4", hq=16, hkv=4, d=64, new=37, caches="5003,1200,64,2777,333,0",
             text=False, fuse=False, f32=True, lse=True, new_lens=""),
        # two long sessions, 512-token blocks over 131072 tokens each
        dict(name="cache4_step_streams", kind="step4", hq=64, hkv=8, d=128, new=512, caches="131072,131072",
             text=False, fuse=True, f32=False, lse=False, new_lens=""),
    ]


HEADS = ((24, 24, 128), (32, 8, 128), (40, 8, 128), (64, 8, 128), (16, 4, 64), (8, 8, 64), (12, 4, 128), (8, 1, 128))
MAX_FLOPS, MAX_BYTES = 4.5e12, 2.0e9   # no drawn case costs more than the largest listed ones


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        hq, hkv, d = rng.choice(HEADS)
        kind = rng.choice(("wstep", "wstep", "wprefill", "wprefill", "wtrain", "wtrain", "append4", "step4", "step4",
                           "step4"))
        heads = dict(hq=hq, hkv=hkv, d=d)
        win = dict(window=_log_int(rng, 16, 16384), sinks=rng.choice((0, 4, 64, _log_int(rng, 1, 512))))
        if kind in ("wstep", "step4", "append4"):
            b = rng.choice((1, 1, 2, 3, 4, 6, 8))
            top = _log_int(rng, 128, 131072)
            # sessions of one age, or of ages spread below the oldest
            same = rng.random() < 0.3
            caches = [top if same or i == 0 else _log_int(rng, 1, top) for i in range(b)]
            rng.shuffle(caches)
            new = rng.choice((1, _log_int(rng, 2, 16), _log_int(rng, 16, 512), _log_int(rng, 64, 512)))
            if kind == "append4":
                new = rng.choice((new, _log_int(rng, 512, 16384)))
            case = dict(kind=kind, new=new, caches=",".join(map(str, caches)), **heads)
            if kind != "append4":
                lens = ""
                if b > 1 and rng.random() < 0.3:
                    lens = ",".join(str(rng.randint(max(1, new // 3), new)) for _ in range(b))
                case.update(text=rng.random() < 0.4, fuse=rng.random() < 0.6, f32=rng.random() < 0.2,
                            lse=rng.random() < 0.3, new_lens=lens)
            if kind == "wstep":
                case.update(win)
        else:
            batch = rng.choice((1, 1, 2, 3))
            blocks = _log_int(rng, 1, 96)
            block = rng.choice((0, 0, _log_int(rng, 16, 512)))
            case = dict(kind=kind, batch=batch, blocks=blocks, block=block, layout=rng.randint(0, 1 << 30),
                        text=block == 0 and rng.random() < 0.5, **heads, **win)
            if kind == "wprefill":
                case.update(paged=rng.random() < 0.5, f32=rng.random() < 0.2, lse=rng.random() < 0.3)
        need = work(case)
        if need["flops"] <= MAX_FLOPS and need["bytes"] <= MAX_BYTES:
            return case


# ---- lengths of a case -----------------------------------------------------

def _ints(text):
    return [int(x) for x in text.split(",") if x]


def _layout(case):
    """Block offsets [B][nb+1] and segment starts [B][nb] (or None): equal
    blocks, or interleaved units (a visual segment of 64..256 tokens, an audio
    one of 4..16, up to 8 text tokens) in another order per stream."""
    nb, b = case["blocks"], case["batch"]
    if case["block"]:
        total, t = [case["block"]] * nb, [0] * nb
    else:
        g = torch.Generator().manual_seed(case["layout"])
        vis, aud, txt = (torch.randint(lo, hi + 1, (nb,), generator=g) for lo, hi in ((64, 256), (4, 16), (0, 8)))
        total, t = (vis + aud + txt).tolist(), txt.tolist()
    off = torch.zeros((b, nb + 1), dtype=torch.int32)
    off[:, 1:] = torch.tensor([total[s % nb:] + total[:s % nb] for s in range(b)], dtype=torch.int32).cumsum(1)
    starts = off[:, 1:] - torch.tensor([t[s % nb:] + t[:s % nb] for s in range(b)], dtype=torch.int32)
    return off, (starts.contiguous() if case["text"] else None)


def _row_ranges(case, off, starts, b):
    """[L], [L]: lo and hi of every token of stream b of a whole sequence."""
    lens = (off[b, 1:] - off[b, :-1]).long()
    pos = torch.arange(int(off[b, -1]))
    first = torch.repeat_interleave(off[b, :-1].long(), lens)
    hi = torch.repeat_interleave(off[b, 1:].long(), lens)
    if starts is not None:
        tau = torch.repeat_interleave(starts[b].long(), lens)
        first = torch.where(pos >= tau, pos, first)
        hi = torch.maximum(tau, pos + 1)
    return first - case["window"], hi


def _step_lens(case):
    """Per stream: cached tokens, new tokens, start of the token-causal
    segment within the new block (a decode block is all segment; a unit ends
    in up to 8 text tokens)."""
    caches = _ints(case["caches"])
    new = case["new"]
    lens = _ints(case.get("new_lens", "")) or [new] * len(caches)
    starts = [0 if new <= 16 else n - 1 - b % 8 for b, n in enumerate(lens)]
    return caches, lens, starts


def _step_ranges(case, b):
    """lo and hi of stream b's real rows, positions counted from the session's
    first token."""
    caches, lens, starts = _step_lens(case)
    t = torch.arange(lens[b])
    tau = starts[b] if case["text"] else lens[b]
    first = torch.where(t >= tau, t, torch.zeros_like(t))
    hi = torch.clamp(torch.maximum(torch.full_like(t, tau), t + 1), max=lens[b])
    if "window" not in case:
        return torch.zeros_like(t), caches[b] + hi
    return caches[b] + first - case["window"], caches[b] + hi


def _pairs(lo, hi, sinks):
    """Visible (row, key) pairs."""
    lo = lo.clamp(min=0)
    return float((hi - lo).sum() + torch.minimum(lo, torch.full_like(lo, sinks)).sum())


# ---- the 4-bit format -------------------------------------------------------

def _quantise(x):
    """Codes (two a byte, the even element in the low half) and scale bytes of
    x [...][d]: [...][d / 2], [...][d / 32] uint8."""
    x = x.float().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True))
    e = torch.clamp(torch.where(m <= 0.75, e - 3, e - 2), -100, 125)
    e = torch.where(m == 0, torch.full_like(e, -100), e)
    y = torch.ldexp(x, -e)
    a = y.abs()
    c = (a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() \
        + (a >= 3.5).int() + (a > 5).int() + 8 * torch.signbit(y).int()
    c = c.reshape(*c.shape[:-2], 16 * c.shape[-2], 2)
    return (c[..., 0] + 16 * c[..., 1]).to(torch.uint8), (e[..., 0] + 127).to(torch.uint8)


def _values(codes, scales):
    """The values codes and scale bytes stand for, f32 (exact in bf16)."""
    c = torch.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1]).long()
    table = torch.tensor((0, .5, 1, 1.5, 2, 3, 4, 6), device=codes.device)
    x = torch.where(c >= 8, -table[c & 7], table[c & 7])
    return torch.ldexp(x.reshape(*scales.shape, 32), scales.int()[..., None] - 127).reshape(x.shape)


# ---- inputs ----------------------------------------------------------------

def _randn(g, shape, scale=1.0):
    x = torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)
    return (x * scale).to(torch.bfloat16)


def _pair(values):
    host = torch.as_tensor(values, dtype=torch.int32).contiguous()
    return host, host.to(DEV)


def _pages(seed, batch, per):
    """A page table whose pages lie in a random physical order, and the pool's size."""
    pages = batch * per + 2
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))[:batch * per]
    return order.reshape(batch, per).to(torch.int32), pages


def _inputs(case, seed):
    """The random tensors of a case."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    hq, hkv, d, kind = case["hq"], case["hkv"], case["d"], case["kind"]
    x = {}
    if kind in ("wstep", "step4", "append4"):
        caches, lens, starts = _step_lens(case)
        b, new = len(caches), case["new"]
        x["k"], x["v"] = _randn(g, (b, new, hkv, d)), _randn(g, (b, new, hkv, d))
        if kind != "append4":
            x["q"] = _randn(g, (b, new, hq, d))
        if kind == "step4":
            # histories; a few channels of the keys are larger than the rest
            wide = torch.ones(d, device=DEV, dtype=torch.bfloat16)
            wide[5::31] = 4
            x["hist"] = [(_randn(g, (c, hkv, d)) * wide, _randn(g, (c, hkv, d))) for c in caches]
        if kind == "wstep":
            # only the pages that some visible or new token lives in exist
            per = -(-(max(caches) + new) // PAGE)
            live = torch.zeros((b, per), dtype=torch.bool)
            for i, c in enumerate(caches):
                live[i, :-(-min(case["sinks"], c) // PAGE)] = True
                live[i, max(0, c - case["window"]) // PAGE:-(-(c + lens[i]) // PAGE)] = True
            pages = int(live.sum()) + 2
            order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))[:pages - 2]
            table = torch.full((b, per), -1, dtype=torch.int32)
            table[live] = order.to(torch.int32)
            x["table"] = table
            x["kpool"], x["vpool"] = _randn(g, (pages, hkv, PAGE, d)), _randn(g, (pages, hkv, PAGE, d))
        return x
    off, _ = _layout(case)
    b, length = case["batch"], int(off[0, -1])
    x["q"] = _randn(g, (b, length, hq, d))
    if case.get("paged"):
        x["table"], pages = _pages(seed, b, -(-length // PAGE))
        x["kpool"], x["vpool"] = _randn(g, (pages, hkv, PAGE, d)), _randn(g, (pages, hkv, PAGE, d))
    else:
        x["k"], x["v"] = _randn(g, (b, length, hkv, d), 0.5), _randn(g, (b, length, hkv, d))
    if kind == "wtrain":
        x["dout"] = _randn(g, (b, length, hq, d))
    return x


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] in ("wstep", "step4", "append4"):
        caches, lens, starts = _step_lens(case)
        s["lens"] = _pair(caches)
        s["new_lens"] = _pair(lens) if case.get("new_lens") else None
        s["starts"] = _pair(starts) if case.get("text") else None
        if own:
            import paper_2606_25041_amd as ws
            if case["kind"] == "wstep":
                s["cache"] = ws.PagedCache(s["kpool"], s["vpool"], s["table"])
            else:
                table, pages = _pages(seed, len(caches), -(-(max(caches) + case["new"]) // PAGE))
                s["cache"] = ws.PagedCache4.allocate(pages, case["hkv"], case["d"], table, device=DEV)
                for b, (hk, hv) in enumerate(s.pop("hist", ())):
                    if hk.shape[0]:
                        one = ws.PagedCache4(s["cache"].pool, table[b:b + 1])
                        ws.kv_append(one, [0], hk[None], hv[None])
        else:
            if case["kind"] == "wstep":
                s["table"] = s["table"].to(DEV)
            elif case["kind"] == "step4":
                s["hist"] = [tuple(_quantise(t) for t in kv) for kv in s["hist"]]
            if case["kind"] != "append4":
                s["ranges"] = [_step_ranges(case, b) for b in range(len(caches))]
        return s
    off, starts = _layout(case)
    s["offsets"] = (off, off.to(DEV))
    s["starts"] = None if starts is None else (starts, starts.to(DEV))
    if own and case.get("paged"):
        import paper_2606_25041_amd as ws
        s["cache"] = ws.PagedCache(s["kpool"], s["vpool"], s["table"])
    if not own:
        if case.get("paged"):
            s["table"] = s["table"].to(DEV)
        s["ranges"] = [_row_ranges(case, off, starts, b) for b in range(case["batch"])]
    return s


# ---- the operators in plain torch --------------------------------------------

def _attend(q, keys, lo, hi, sinks, dout=None, f=torch.float32):
    """q [R][Hq][d]; keys(p): the keys and values [n][Hkv][d] at positions p.
    Row t sees positions < hi[t] that are < sinks or >= lo[t] (both
    non-decreasing).  Returns out [R][Hq][d], lse [Hq][R] and, given dout, dq
    and a list of (positions, dk, dv) parts, [n][Hkv][d]."""
    rows, hq, d = q.shape
    scale = 1.0 / math.sqrt(d)
    out = torch.empty((rows, hq, d), dtype=f, device=q.device)
    lse = torch.empty((hq, rows), dtype=f, device=q.device)
    dq, parts = torch.empty_like(out) if dout is not None else None, []
    step = rows
    while step > 64 and hq * step * (int(hi[min(step, rows) - 1]) - max(int(lo[0]), 0) + sinks) > 1 << 28:
        step = -(-step // 2)
    for a in range(0, rows, step):
        e = min(rows, a + step)
        low, top = max(int(lo[a]), 0), int(hi[e - 1])
        p = torch.cat((torch.arange(0, min(sinks, low)), torch.arange(low, top))).to(q.device)
        k, v = (x.to(f).transpose(0, 1).contiguous() for x in keys(p))     # [Hkv][n][d]
        hkv = k.shape[0]
        g = hq // hkv

        def heads(x):   # [e - a][Hq][d] -> [Hkv][G (e - a)][d]
            return x[a:e].to(f).reshape(e - a, hkv, g, d).permute(1, 2, 0, 3).reshape(hkv, g * (e - a), d)

        def rows_of(x):
            return x.reshape(hkv, g, e - a, d).permute(2, 0, 1, 3).reshape(e - a, hq, d)

        qh = heads(q)
        s = (torch.bmm(qh, k.transpose(1, 2).contiguous()) * scale).reshape(hkv, g, e - a, -1)
        l_, h_ = lo[a:e].to(q.device)[:, None], hi[a:e].to(q.device)[:, None]
        s = s.masked_fill(~((p < h_) & ((p < sinks) | (p >= l_))), -math.inf)
        m = s.amax(-1, keepdim=True)
        w = torch.exp(s - m)
        z = w.sum(-1, keepdim=True)
        w = (w / z).reshape(hkv, g * (e - a), -1)
        o = torch.bmm(w, v)
        out[a:e] = rows_of(o)
        lse[:, a:e] = (m + torch.log(z))[..., 0].reshape(hq, e - a)
        if dout is not None:
            do = heads(dout)
            ds = torch.bmm(do, v.transpose(1, 2).contiguous())
            ds = w * (ds - (do * o).sum(-1, keepdim=True))
            dq[a:e] = rows_of(torch.bmm(ds, k) * scale)
            parts.append((p, (torch.bmm(ds.transpose(1, 2).contiguous(), qh) * scale).transpose(0, 1),
                          torch.bmm(w.transpose(1, 2).contiguous(), do).transpose(0, 1)))
    return out, lse, dq, parts


def _paged(s, b):
    """Keys and values of stream b's cache at positions p."""
    def at(p):
        page, slot = s["table"][b].long()[p // PAGE], p % PAGE
        return s["kpool"][page, :, slot], s["vpool"][page, :, slot]
    return at


def _step_keys(s, b):
    case = s["case"]
    caches, lens, _ = _step_lens(case)
    n = caches[b]
    if case["kind"] == "wstep":
        cached = _paged(s, b)
    else:
        (kc, ks), (vc, vs) = s["hist"][b]

        def cached(p):
            return _values(kc[p], ks[p]), _values(vc[p], vs[p])

    def at(p):
        old = p[p < n]
        new = p[p >= n] - n
        return tuple(torch.cat((c.to(x.dtype) if case["kind"] == "wstep" else c, x[b, new].to(c.dtype)))
                     for c, x in zip(cached(old), (s["k"], s["v"])))
    return at


def _plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "append4":
        return {"k": _values(*_quantise(s["k"])).to(torch.bfloat16), "v": _values(*_quantise(s["v"])).to(torch.bfloat16)}
    sinks = case.get("sinks", 0)
    if kind in ("wstep", "step4"):
        caches, lens, _ = _step_lens(case)
        got = [_attend(s["q"][b, :n], _step_keys(s, b), *s["ranges"][b], sinks)[:2] for b, n in enumerate(lens)]
        dt = torch.float32 if case["f32"] else torch.bfloat16
        res = {"out": [o.to(dt) for o, _ in got]}
        if case["lse"]:
            res["lse"] = [l for _, l in got]
        if case["fuse"] and kind == "wstep":
            for b, (c, n) in enumerate(zip(caches, lens)):
                p = torch.arange(c, c + n, device=DEV)
                page = s["table"][b].long()[p // PAGE]
                s["kpool"][page, :, p % PAGE] = s["k"][b, :n]
                s["vpool"][page, :, p % PAGE] = s["v"][b, :n]
            res["k_pool"], res["v_pool"] = s["kpool"], s["vpool"]
        elif case["fuse"]:
            res["k"], res["v"] = (_values(*_quantise(x)).to(torch.bfloat16) for x in (s["k"], s["v"]))
            if s["new_lens"] is not None:
                res["k"], res["v"] = ([x[b, :n] for b, n in enumerate(lens)] for x in (res["k"], res["v"]))
        return res
    outs = []
    for b in range(case["batch"]):
        if case.get("paged"):
            keys = _paged(s, b)
        else:
            def keys(p, b=b):
                return s["k"][b, p], s["v"][b, p]
        outs.append(_attend(s["q"][b], keys, *s["ranges"][b], sinks, s["dout"][b] if kind == "wtrain" else None))
    out = torch.stack([o[0] for o in outs]).to(torch.float32 if case.get("f32") else torch.bfloat16)
    res = {"out": out}
    if case.get("lse") or kind == "wtrain":
        res["lse"] = torch.stack([o[1] for o in outs])
    if kind == "wtrain":
        # bf16 gradients, as bf16 training takes them
        res["dq"] = torch.stack([o[2] for o in outs]).to(torch.bfloat16)
        for i, name in ((1, "dk"), (2, "dv")):
            total = torch.zeros(s["k"].shape, dtype=torch.float32, device=DEV)
            for b, o in enumerate(outs):
                for part in o[3]:
                    total[b].index_add_(0, part[0], part[i])
            res[name] = total.to(torch.bfloat16)
    return res


# ---- one pass --------------------------------------------------------------

def run(s):
    if not own:
        return _plain(s)
    import paper_2606_25041_amd as ws
    case, kind = s["case"], s["case"]["kind"]
    if kind == "append4":
        ws.kv_append(s["cache"], s["lens"], s["k"], s["v"])
        k, v = ws.kv_read(s["cache"], s["lens"], case["new"])
        return {"k": k, "v": v}
    if kind in ("wstep", "step4"):
        win = dict(window=case["window"], sinks=case["sinks"]) if kind == "wstep" else {}
        got = ws.block_causal_attn_fwd(s["q"], s["k"], s["v"], s["cache"], s["lens"], fuse_append=case["fuse"],
                                       out_dtype=torch.float32 if case["f32"] else torch.bfloat16,
                                       want_lse=case["lse"], text_starts=s["starts"], new_lens=s["new_lens"], **win)
        out, lse = got if case["lse"] else (got, None)
        lens = _step_lens(case)[1]
        res = {"out": [out[b, :n] for b, n in enumerate(lens)]}   # padding rows are unspecified
        if case["lse"]:
            res["lse"] = [lse[b, :, :n] for b, n in enumerate(lens)]
        if case["fuse"] and kind == "wstep":
            res["k_pool"], res["v_pool"] = s["cache"].k_pool, s["cache"].v_pool
        elif case["fuse"]:
            res["k"], res["v"] = ws.kv_read(s["cache"], s["lens"], case["new"])
            if s["new_lens"] is not None:
                res["k"], res["v"] = ([x[b, :n] for b, n in enumerate(lens)] for x in (res["k"], res["v"]))
        return res
    win = dict(text_starts=s["starts"], window=case["window"], sinks=case["sinks"])
    if kind == "wprefill":
        got = ws.block_causal_prefill(s["q"], s.get("k"), s.get("v"), s["offsets"], cache=s.get("cache"),
                                      out_dtype=torch.float32 if case["f32"] else torch.bfloat16,
                                      want_lse=case["lse"], **win)
        return {"out": got[0], "lse": got[1]} if case["lse"] else {"out": got}
    out, lse = ws.block_causal_prefill(s["q"], s["k"], s["v"], s["offsets"], want_lse=True, **win)
    dq, dk, dv = ws.block_causal_prefill_bwd(s["q"], s["k"], s["v"], out, s["dout"], lse, s["offsets"],
                                             grad_dtype=torch.bfloat16, **win)
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


# ---- what a pass cannot do without ------------------------------------------

def work(case):
    hq, hkv, d, kind = case["hq"], case["hkv"], case["d"], case["kind"]
    sinks = case.get("sinks", 0)
    row4 = 2.0 * hkv * (d // 2 + d // 32)     # a token's keys and values at 4 bits
    if kind in ("wstep", "step4", "append4"):
        caches, lens, _ = _step_lens(case)
        new = sum(lens)
        if kind == "append4":   # bf16 in, 4 bits out, and the values read back
            return {"bytes": new * (8.0 * hkv * d + 2 * row4), "flops": 0.0}
        ranges = [_step_ranges(case, b) for b in range(len(caches))]
        pairs = sum(_pairs(lo, hi, sinks) for lo, hi in ranges)
        row = row4 if kind == "step4" else 4.0 * hkv * d
        live = 0
        for (lo, _), n in zip(ranges, caches):
            low = max(int(lo[0]), 0)
            live += min(sinks, low) + n - min(low, n)
        io = new * hq * d * (2.0 + (4.0 if case["f32"] else 2.0)) + (4.0 * new * hq if case["lse"] else 0.0)
        commit = 0.0
        if case["fuse"]:
            commit = new * (2 * row + 4.0 * hkv * d if kind == "step4" else row)
        return {"bytes": live * row + 4.0 * new * hkv * d + io + commit, "flops": 4.0 * d * hq * pairs}
    off, starts = _layout(case)
    b, length = case["batch"], int(off[0, -1])
    pairs = sum(_pairs(*_row_ranges(case, off, starts, i), sinks) for i in range(b))
    q, kv = 1.0 * b * length * hq * d, 2.0 * b * length * hkv * d
    if kind == "wprefill":
        lse = 4.0 * b * length * hq if case["lse"] else 0.0
        return {"bytes": 2 * q + 2 * kv + q * (4 if case["f32"] else 2) + lse, "flops": 4.0 * d * hq * pairs}
    # forward (q, k, v -> out, lse) and gradients (dout -> dq, dk, dv)
    return {"bytes": 2 * q + 2 * kv + 2 * q + 2 * q + 2 * q + 2 * kv + 4.0 * b * length * hq,
            "flops": 14.0 * d * hq * pairs}


# ---- the same in 64 bits, row by row from the definition ----------------------

E2M1 = [(-1) ** (c >> 3) * (0, .5, 1, 1.5, 2, 3, 4, 6)[c & 7] for c in range(16)]


def _rounded4(x):
    """x as the 4-bit cache returns it, in 64 bits: the nearest of the sixteen
    values by distance, ties to the even code."""
    y = x.double().reshape(-1, 32)
    top = y.abs().amax(1, keepdim=True)
    e = torch.full_like(top, -100)
    for _ in range(226):   # the least exponent that holds the largest value
        grow = (top > 6 * torch.pow(2.0, e)) & (e < 125)
        if not bool(grow.any()):
            break
        e = torch.where(grow, e + 1, e)
    y = y / torch.pow(2.0, e)
    best, dist = torch.zeros_like(y), torch.full_like(y, math.inf)
    for c in (0, 2, 4, 6, 1, 3, 5, 7):   # even codes first: they keep a tie
        near = (y.abs() - E2M1[c]).abs()
        take = near < dist
        best, dist = torch.where(take, torch.full_like(y, E2M1[c]), best), torch.minimum(near, dist)
    return (torch.where(y < 0, -best, best) * torch.pow(2.0, e)).reshape(x.shape)


def _exact_rows(case, q, k, v, b, base, dout=None):
    """Stream b's rows at positions base.. over all keys k, v [N][Hkv][d] (those
    that no row sees may hold anything finite)."""
    rows, hq, d = q.shape
    n, hkv = k.shape[:2]
    g = hq // hkv
    lo, hi = (x.to(q.device) for x in (_step_ranges(case, b) if "caches" in case
                                       else _row_ranges(case, *_layout(case), b)))
    sinks = case.get("sinks", 0)
    out = torch.empty((rows, hq, d), dtype=torch.float64, device=q.device)
    lse = torch.empty((hq, rows), dtype=torch.float64, device=q.device)
    dq = torch.empty_like(out)
    dk, dv = (torch.zeros((n, hkv, d), dtype=torch.float64, device=q.device) for _ in range(2))
    step = max(1, (1 << 27) // max(n, 1))
    j = torch.arange(n, device=q.device)[None]
    for a in range(0, rows, step):
        e = min(rows, a + step)
        top = int(hi[e - 1])
        see = (j < hi[a:e, None]) & ((j < sinks) | (j >= lo[a:e, None]))
        see = see[:, :top]
        for h in range(hq):
            kh, vh = k[:top, h // g].double(), v[:top, h // g].double()
            qh = q[a:e, h].double() / math.sqrt(d)
            s = torch.where(see, qh @ kh.t().contiguous(), -math.inf)
            l = torch.logsumexp(s, 1)
            w = torch.exp(s - l[:, None])
            o = w @ vh
            out[a:e, h], lse[h, a:e] = o, l
            if dout is not None:
                do = dout[a:e, h].double()
                ds = w * (do @ vh.t().contiguous() - (do * o).sum(1, keepdim=True))
                dq[a:e, h] = ds @ kh / math.sqrt(d)
                dk[:top, h // g] += ds.t().contiguous() @ qh
                dv[:top, h // g] += w.t().contiguous() @ do
    return out, lse, dq, dk, dv


def exact(case, seed):
    x = _inputs(case, seed)
    kind, d, hkv = case["kind"], case["d"], case["hkv"]
    if kind == "append4":
        return {"k": _rounded4(x["k"]), "v": _rounded4(x["v"])}
    if kind in ("wstep", "step4"):
        caches, lens, _ = _step_lens(case)
        outs, lses = [], []
        for b, (c, n) in enumerate(zip(caches, lens)):
            if kind == "step4":
                old = [_rounded4(t) for t in x["hist"][b]]
            else:   # positions without a page hold zeros, which no row sees
                p = torch.arange(c, device=DEV)
                page = x["table"][b].to(DEV).long()[p // PAGE]
                old = [torch.where((page >= 0)[:, None, None], t[page.clamp(min=0), :, p % PAGE], 0) for t in
                       (x["kpool"], x["vpool"])]
            k, v = (torch.cat((o, t[b, :n].to(o.dtype))) for o, t in zip(old, (x["k"], x["v"])))
            o, l = _exact_rows(case, x["q"][b, :n], k, v, b, c)[:2]
            outs.append(o)
            lses.append(l)
        res = {"out": outs}
        if case["lse"]:
            res["lse"] = lses
        if case["fuse"] and kind == "wstep":   # copies: nothing is computed
            res["k_pool"] = res["v_pool"] = None
        elif case["fuse"]:
            res["k"], res["v"] = _rounded4(x["k"]), _rounded4(x["v"])
            if case["new_lens"]:
                res["k"], res["v"] = ([t[b, :n] for b, n in enumerate(lens)] for t in (res["k"], res["v"]))
        return res
    got = []
    for b in range(case["batch"]):
        if case.get("paged"):
            p = torch.arange(x["q"].shape[1], device=DEV)
            page = x["table"][b].to(DEV).long()[p // PAGE]
            k, v = x["kpool"][page, :, p % PAGE], x["vpool"][page, :, p % PAGE]
        else:
            k, v = x["k"][b], x["v"][b]
        got.append(_exact_rows(case, x["q"][b], k, v, b, 0, x["dout"][b] if kind == "wtrain" else None))
    names = ["out"] + (["lse"] if case.get("lse") or kind == "wtrain" else [])
    names += ["dq", "dk", "dv"] if kind == "wtrain" else []
    at = dict(out=0, lse=1, dq=2, dk=3, dv=4)
    return {n: torch.stack([r[at[n]] for r in got]) for n in names}
