"""What the windowed and the 4-bit entry points refuse, on the CPU: every status
of the C ABI before anything is enqueued (all device pointers are fake and never
dereferenced), and the Python arguments that have no meaning."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2606_25041_amd as ws

if torch.cuda.device_count() > 0:
    pytest.skip("uses fake device pointers; CPU-only module", allow_module_level=True)

FAKE = 0x10000
OK, NULL, SHAPE, UNSUPPORTED, ALIGN, OFFSETS, PAGE, CAPACITY, HEADS, WORKSPACE, HIP = range(11)


@pytest.fixture(scope="module")
def lib():
    return ws.library()


def t4(ptr=FAKE, dtype=ws.WS_DTYPE_BF16, d=128, L=16, H=4, **kw):
    s = dict(sb=L * H * d, st=H * d, sh=d)
    s.update(kw)
    return ws.Tensor4(ptr, dtype, s["sb"], s["st"], s["sh"])


class Host:
    def __init__(self, lens=(10, 100), new=(16, 3), text=(0, 16), max_pages=4, num_pages=10):
        self.lens, self.new, self.text = (np.array(x, np.int32) for x in (lens, new, text))
        self.table = np.arange(2 * max_pages, dtype=np.int32).reshape(2, max_pages) % num_pages
        self.max_pages, self.num_pages = max_pages, num_pages

    def desc(self, four, **kw):
        d = dict(page_table_dev=FAKE, page_table_host=self.table.ctypes.data, num_pages=self.num_pages, page_size=64,
                 max_pages_per_seq=self.max_pages, num_kv_heads=2, head_dim=128)
        d.update(dict(pool=FAKE) if four else dict(k_pool=FAKE, v_pool=FAKE))
        d.update(kw)
        return (ws.PagedKV4Desc if four else ws.PagedKVDesc)(**d)


def step(lib, h, four, desc=None, q=None, kn=None, vn=None, out=None, B=2, Lq=16, Hq=4, sinks=4, window=64, scale=0.1,
         flags=0, lse=None, lens="host", new=(None, None), text=(None, None), null_desc=False):
    desc = desc or h.desc(four)
    args = [q or t4(H=Hq, L=Lq), kn or t4(H=2, L=Lq), vn or t4(H=2, L=Lq), None if null_desc else ctypes.byref(desc),
            h.lens.ctypes.data if lens == "host" else lens, FAKE, *new, *text, B, Lq, Hq]
    tail = [scale, flags, out or t4(H=Hq, L=Lq), lse, FAKE, 1 << 40, None]
    if four:
        return lib.ws_block_causal_attn_fwd_4bit(*args, *tail)
    return lib.ws_block_causal_attn_fwd_window(*args, sinks, window, *tail)


@pytest.mark.parametrize("four", (False, True))
def test_step_refusals(lib, four):
    h = Host()
    c = lambda **kw: step(lib, h, four, **kw)  # noqa: E731
    assert c() == HIP and b"compute units" in lib.ws_last_error()   # valid: reaches the device plan
    assert c(B=0) == OK and c(Lq=0) == OK
    assert c(B=0, q=ws.Tensor4(None, 1, 0, 0, 0)) == OK
    for kw in (dict(q=t4(None)), dict(kn=t4(None)), dict(out=t4(None)), dict(lens=None), dict(null_desc=True),
               dict(desc=h.desc(four, page_table_host=None)), dict(desc=h.desc(four, page_table_dev=None)),
               dict(desc=h.desc(four, **({"pool": None} if four else {"v_pool": None}))),
               dict(new=(h.new.ctypes.data, None)), dict(new=(None, FAKE)), dict(text=(h.text.ctypes.data, None)),
               dict(text=(None, FAKE))):
        assert c(**kw) == NULL, kw
    for kw in (dict(B=-1), dict(Lq=-1), dict(Hq=0), dict(kn=t4(H=2, st=1 << 24, sb=1 << 24)),
               dict(vn=t4(H=2, st=1 << 24, sb=1 << 24)), dict(q=t4(sh=-128)),
               dict(desc=h.desc(four, num_pages=0)), dict(desc=h.desc(four, max_pages_per_seq=-1))):
        assert c(**kw) == SHAPE, kw
    for kw in (dict(q=t4(dtype=ws.WS_DTYPE_F32)), dict(kn=t4(dtype=ws.WS_DTYPE_F32)), dict(flags=2), dict(scale=0.0),
               dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")),
               dict(desc=h.desc(four, head_dim=96)), dict(desc=h.desc(four, page_size=32)), dict(out=t4(dtype=3))):
        assert c(**kw) == UNSUPPORTED, kw
    for kw in (dict(q=t4(FAKE + 2)), dict(kn=t4(H=2, sh=132)), dict(lse=FAKE + 2), dict(out=t4(FAKE + 8)),
               dict(desc=h.desc(four, **({"pool": FAKE + 8} if four else {"k_pool": FAKE + 8})))):
        assert c(**kw) == ALIGN, kw
    assert c(Hq=3) == HEADS
    for bad, want in ((Host(lens=(10, -1)), SHAPE), (Host(lens=(10, 300)), CAPACITY), (Host(max_pages=2, lens=(10, 129)), CAPACITY)):
        assert step(lib, bad, four, window=1 << 20) == want
    assert step(lib, Host(lens=(10, 250)), four, flags=ws.WS_FUSE_APPEND) == CAPACITY   # the commit does not fit
    h2 = Host()
    h2.table[1, 1] = 10
    assert step(lib, h2, four, window=1 << 20) == PAGE
    for new in ((0, 3), (17, 3)):
        h3 = Host(new=new)
        assert step(lib, h3, four, new=(h3.new.ctypes.data, FAKE)) == SHAPE
    for text in ((-1, 0), (0, 17)):
        h3 = Host(text=text)
        assert step(lib, h3, four, text=(h3.text.ctypes.data, FAKE)) == OFFSETS
    assert step(lib, h, four, new=(h.new.ctypes.data, FAKE), text=(h.text.ctypes.data, FAKE)) == HIP


def test_windows_must_not_be_negative(lib):
    h = Host()
    assert step(lib, h, False, sinks=-1) == SHAPE and step(lib, h, False, window=-1) == SHAPE
    assert step(lib, h, False, sinks=2 ** 31 - 1, window=2 ** 31 - 1) == HIP
    assert lib.ws_step_workspace_bytes_window(2, 4, 2, 16, h.lens.ctypes.data, None, -1, 4) == 0
    assert lib.ws_prefill_window_bwd_workspace_bytes(1, 4, 2, 16, 0, -1) == 0
    assert lib.ws_prefill_window_bwd_workspace_bytes(1, 4, 3, 16, 0, 1) == 0
    # two heads' rows: lse and D of 4 x 16 rows rounded up to 256 bytes, then two entries a token
    assert lib.ws_prefill_window_bwd_workspace_bytes(1, 4, 2, 16, 0, 1) >= 512 + 2 * 4 * 16


def _sequence(lib, bwd, off, B=1, L=16, nb=None, sinks=0, window=4, text=(None, None), lse=FAKE, scale=0.1, d=128, Hq=4,
              Hkv=2, wsb=1 << 40, **kw):
    off = np.ascontiguousarray(off, np.int32)
    nb = off.shape[-1] - 1 if nb is None else nb
    q = kw.get("q") or t4(H=Hq, L=L, d=d)
    k, v = (kw.get(n) or t4(H=Hkv, L=L, d=d) for n in "kv")
    out = kw.get("out") or t4(H=Hq, L=L, d=d)
    head = [off.ctypes.data if kw.get("offsets", True) else None, FAKE, *text, B, L, nb, Hq, Hkv, d, sinks, window, scale]
    if bwd:
        g = [kw.get(n) or t4(H=Hq if n == "dq" else Hkv, L=L, d=d) for n in ("dq", "dk", "dv")]
        return lib.ws_block_causal_prefill_window_bwd(q, k, v, out, out, lse, *head, *g, FAKE, wsb, None)
    return lib.ws_block_causal_prefill_window(q, k, v, None, *head, out, None, None)


@pytest.mark.parametrize("bwd", (False, True))
def test_sequence_refusals(lib, bwd):
    c = lambda off=((0, 7, 16),), **kw: _sequence(lib, bwd, off, **kw)  # noqa: E731
    assert c(B=0) == OK and c(off=((0, 0),), L=0) == OK
    for kw in (dict(q=t4(None)), dict(k=t4(None)), dict(out=t4(None)), dict(offsets=False), dict(text=(FAKE, None)),
               dict(text=(None, FAKE))):
        assert c(**kw) == NULL, kw
    for kw in (dict(B=-1), dict(L=-1), dict(Hq=0), dict(Hkv=0), dict(sinks=-1), dict(window=-1)):
        assert c(**kw) == SHAPE, kw
    for kw in (dict(d=96), dict(scale=0.0), dict(scale=float("nan")), dict(q=t4(dtype=ws.WS_DTYPE_F32))):
        assert c(**kw) == UNSUPPORTED, kw
    for off in (((1, 7, 16),), ((0, 9, 7),), ((0, 7, 15),), ((0, 7, 17),)):
        assert c(off=off) == OFFSETS, off
    text = np.array([[8, 16]], np.int32)   # outside its block [0, 7]
    assert c(text=(text.ctypes.data, FAKE)) == OFFSETS
    assert c(Hq=3) == HEADS
    assert c(q=t4(FAKE + 4)) == ALIGN
    if bwd:
        assert c(lse=None) == NULL and c(lse=FAKE + 2) == ALIGN
        assert c(dq=t4(dtype=ws.WS_DTYPE_F32)) == UNSUPPORTED   # mixed dtypes
        assert c(dv=t4(dtype=ws.WS_DTYPE_F32, H=2)) == UNSUPPORTED
        assert c(wsb=512 + 2 * 4 * 16 - 1) == WORKSPACE


def test_4bit_append_and_read_refusals(lib):
    h = Host()

    def append(B=2, L=16, desc=None, k=None, lens="host", new=(None, None)):
        return lib.ws_kv_append_4bit(ctypes.byref(desc or h.desc(True)), B, h.lens.ctypes.data if lens == "host" else lens,
                                     FAKE, *new, L, k or t4(H=2, L=L), t4(H=2, L=L), None)

    def read(B=2, L=16, desc=None, k=None, lens="host"):
        return lib.ws_kv_read_4bit(ctypes.byref(desc or h.desc(True)), B, h.lens.ctypes.data if lens == "host" else lens,
                                   FAKE, L, k or t4(H=2, L=L), t4(H=2, L=L), None)
    for f in (append, read):
        assert f(B=0) == OK and f(L=0) == OK
        assert f(k=t4(None)) == NULL and f(lens=None) == NULL and f(desc=h.desc(True, pool=None)) == NULL
        assert f(B=-1) == SHAPE and f(L=-1) == SHAPE and f(B=65536) == SHAPE
        assert f(desc=h.desc(True, head_dim=32)) == UNSUPPORTED and f(k=t4(dtype=ws.WS_DTYPE_F32)) == UNSUPPORTED
        assert f(k=t4(FAKE + 8)) == ALIGN
        assert f(L=200) == CAPACITY
        h.table[1, 1] = 10
        assert f() == PAGE
        h.table[1, 1] = 5
        h.lens[0] = -1
        assert f() == SHAPE
        h.lens[0] = 2 ** 31 - 140   # (with 16 tokens: past 2^31 - 129)
        assert f(desc=h.desc(True, max_pages_per_seq=1 << 26)) == SHAPE
        h.lens[0] = 10
    assert append(new=(h.new.ctypes.data, None)) == NULL
    h.new[0] = 17
    assert append(new=(h.new.ctypes.data, FAKE)) == SHAPE
    h.new[:] = 0   # nothing to commit: a bad page is not touched
    h.table[:] = -1
    assert append(new=(h.new.ctypes.data, FAKE)) in (OK, HIP)


def test_python_refusals():
    pool = torch.zeros(3, 2, 68 * 64, dtype=torch.uint8)
    table = torch.zeros(1, 3, dtype=torch.int32)
    cache = ws.PagedCache4(pool, table)
    assert (cache.num_pages, cache.num_kv_heads, cache.head_dim) == (3, 2, 64)
    for bad in (pool.to(torch.int8), pool[:, :, 1:], pool[0], pool.transpose(0, 1)):
        with pytest.raises(ValueError):
            ws.PagedCache4(bad, table)
    q, k = torch.zeros(1, 4, 4, 64, dtype=torch.bfloat16), torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16)
    full = ws.PagedCache(torch.zeros(3, 2, 64, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, 64, dtype=torch.bfloat16), table)
    off = torch.tensor([[0, 4]], dtype=torch.int32)
    lse = torch.zeros(1, 4, 4)
    for call in (
            lambda: ws.block_causal_attn_fwd(q, k, k, cache, [0], window=4),             # not over a 4-bit cache
            lambda: ws.block_causal_attn_fwd(q, k, k, full, [0], sinks=4),               # sinks without a window
            lambda: ws.block_causal_attn_fwd(q, k, k, full, [0], window=-1),
            lambda: ws.block_causal_attn_fwd(q, k, k, full, [0], window=2 ** 31),
            lambda: ws.block_causal_attn_fwd(q, k, k, full, [0], window=4, sinks=-1),
            lambda: ws.block_causal_attn_fwd_noalloc(q, k, k, cache, (torch.zeros(1, dtype=torch.int32),) * 2, q),
            lambda: ws.block_causal_prefill(q, None, None, off, cache=cache),
            lambda: ws.block_causal_prefill(q, k, k, off, sinks=1),
            lambda: ws.block_causal_prefill_bwd(q, k, k, q, q, lse, off, grad_dtype=torch.bfloat16),
            lambda: ws.block_causal_prefill_bwd(q, k, k, q, q, lse, off, window=4, grad_dtype=torch.float16),
            lambda: ws.kv_read(full, [0], 1),
            lambda: ws.kv_read(cache, [0], -1),
            lambda: ws.block_causal_attn_fwd(q, k, k, cache, [0]),                       # host tensors
            lambda: ws.kv_append(cache, [0], k, k),
            lambda: ws.block_causal_prefill(q, k, k, off, window=4)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        ws.block_causal_prefill(q, k, k, off, window=1.5)
