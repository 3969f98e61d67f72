"""What the linear entry points refuse, on the CPU: every status of the C ABI before
anything is enqueued (device pointers are fake and never dereferenced), workspace
sizes, and the Python arguments that have no meaning."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2606_25041_amd as ws
from paper_2606_25041_amd import linear, packed

if torch.cuda.device_count() > 0:
    pytest.skip("uses fake device pointers; CPU-only module", allow_module_level=True)

FAKE = 0x10000
OK, NULL, SHAPE, UNSUPPORTED, ALIGN, OFFSETS, PAGE, CAPACITY, HEADS, WORKSPACE, HIP = range(11)


@pytest.fixture(scope="module")
def lib():
    return ws.library()


def t3(ptr=FAKE, dtype=ws.WS_DTYPE_BF16, h=4, d=128, **kw):
    s = dict(sb=0, st=h * d, sh=d)
    s.update(kw)
    return ws.Tensor4(ptr, dtype, s["sb"], s["st"], s["sh"])


def state(slots, pool=FAKE, dev=FAKE, num=8, heads=2, d=128):
    host = np.array(slots, np.int32)
    desc = linear.LinearStateDesc(pool, dev, host.ctypes.data if slots is not None else None, num, heads, d)
    desc.keep = host
    return desc


def prefill(lib, off=(0, 5, 9), T=9, S=2, q=None, k=None, v=None, ld=FAKE, hq=4, hkv=2, d=128, scale=0.1, st=None, flags=0,
            out=None, wsp=FAKE, size=1 << 40, off_host="host", off_dev=FAKE):
    host = np.array(off, np.int32)
    return lib.ws_linear_attn_prefill(q or t3(h=hq), k or t3(h=hkv), v or t3(h=hkv), ld, host.ctypes.data if off_host else None,
                                      off_dev, S, T, hq, hkv, d, scale, ctypes.byref(st) if st else None, flags,
                                      out or t3(h=hq), wsp, size, None)


def test_prefill_refusals(lib):
    c = lambda **kw: prefill(lib, **kw)  # noqa: E731
    assert c() == HIP   # valid: reaches the launch, and there is no device
    assert c(st=state((1, 0))) == HIP and c(out=t3(dtype=ws.WS_DTYPE_F32)) == HIP
    assert c(S=0) == OK
    assert c(off=(0, 0, 0)) == OK and c(off=(0, 0, 0), q=t3(ptr=0), k=t3(ptr=0), v=t3(ptr=0), out=t3(ptr=0)) == OK
    assert c(S=-1) == SHAPE and c(T=-1) == SHAPE and c(hq=0) == SHAPE and c(hkv=0) == SHAPE and c(T=2 ** 31 - 1) == SHAPE
    assert c(hkv=70000, hq=70000) == SHAPE
    assert c(hq=5) == HEADS and c(d=96) == UNSUPPORTED
    assert c(off=(1, 5, 9)) == OFFSETS and c(off=(0, 6, 5)) == OFFSETS and c(off=(0, 5, 10)) == OFFSETS
    assert c(off_host=None) == NULL and c(off_dev=None) == NULL and c(ld=None) == NULL and c(ld=FAKE + 2) == ALIGN
    for name in "qkv":
        h = 4 if name == "q" else 2
        assert c(**{name: t3(ptr=0, h=h)}) == NULL
        assert c(**{name: t3(dtype=ws.WS_DTYPE_F32, h=h)}) == UNSUPPORTED
        assert c(**{name: t3(ptr=FAKE + 8, h=h)}) == ALIGN and c(**{name: t3(sh=132, h=h)}) == ALIGN
        assert c(**{name: t3(st=1 << 24, h=h)}) == SHAPE and c(**{name: t3(st=-512, h=h)}) == SHAPE
    assert c(out=t3(ptr=0)) == NULL and c(out=t3(dtype=7)) == UNSUPPORTED and c(out=t3(ptr=FAKE + 4)) == ALIGN
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert c(scale=scale) == UNSUPPORTED
    assert c(flags=4) == UNSUPPORTED
    assert c(wsp=None) == WORKSPACE and c(size=15) == WORKSPACE and c(wsp=FAKE + 8) == WORKSPACE
    need = lib.ws_linear_workspace_bytes(2, 9, 4, 2, 128)
    assert c(size=need) == HIP and c(size=need - 1) == WORKSPACE


def test_state_refusals(lib):
    c = lambda st, **kw: prefill(lib, st=st, **kw)  # noqa: E731
    assert c(state((1, 0), pool=None)) == NULL and c(state((1, 0), dev=None)) == NULL
    assert c(state((1, 0), pool=FAKE + 4)) == ALIGN and c(state((1, 0), num=0)) == SHAPE
    assert c(state((1, 0), heads=4)) == HEADS and c(state((1, 0), d=64)) == HEADS
    assert c(state((1, 8))) == PAGE and c(state((-1, 2))) == PAGE
    assert c(state((3, 3))) == PAGE                                  # written twice
    assert c(state((3, 3)), flags=linear.WS_STATE_KEEP) == HIP       # only read
    assert c(state((99999, 99999), num=100000)) == PAGE and c(state((99999, 99998), num=100000)) == HIP


def step(lib, st=None, q=None, k=None, v=None, ld=FAKE, nl=None, nl_dev="as host", B=2, n=3, hq=4, scale=0.1, flags=0, out=None):
    host = None if nl is None else np.array(nl, np.int32)
    st = state((1, 0)) if st is None else st
    dev = (None if nl is None else FAKE) if nl_dev == "as host" else nl_dev
    return lib.ws_linear_attn_step(q or t3(), k or t3(h=2), v or t3(h=2), ld, ctypes.byref(st) if st else None,
                                   None if host is None else host.ctypes.data, dev, B, n, hq, scale, flags, out or t3(), None)


def test_step_refusals(lib):
    c = lambda **kw: step(lib, **kw)  # noqa: E731
    assert c() == HIP and c(nl=(0, 3)) == HIP and c(flags=linear.WS_STATE_KEEP) == HIP
    assert c(B=0) == OK and c(n=0) == OK
    assert c(st=False) == NULL and c(ld=None) == NULL and c(nl_dev=FAKE) == NULL
    assert c(B=-1) == SHAPE and c(n=-1) == SHAPE and c(hq=0) == SHAPE and c(hq=5) == HEADS
    assert c(nl=(0, 4)) == SHAPE and c(nl=(-1, 2)) == SHAPE
    assert c(flags=linear.WS_STATE_RESET) == UNSUPPORTED and c(scale=0.0) == UNSUPPORTED
    assert c(st=state((1, 1))) == PAGE and c(st=state((1, 8))) == PAGE and c(st=state((1, 0), d=96)) == UNSUPPORTED
    assert c(st=state((1, 1)), flags=linear.WS_STATE_KEEP) == HIP
    assert c(q=t3(ptr=0)) == NULL and c(k=t3(dtype=ws.WS_DTYPE_F32)) == UNSUPPORTED and c(v=t3(sh=4)) == ALIGN
    assert c(out=t3(ptr=FAKE + 2)) == ALIGN


def bwd(lib, off=(0, 5, 9), T=9, S=2, hq=4, hkv=2, d=128, scale=0.1, st=None, ds=None, ds0=None, wsp=FAKE, size=1 << 40, ld=FAKE, **t):
    host = np.array(off, np.int32)
    g = lambda name, h: t.get(name) or t3(h=h)  # noqa: E731
    return lib.ws_linear_attn_prefill_bwd(g("q", hq), g("k", hkv), g("v", hkv), g("dout", hq), ld, host.ctypes.data, FAKE, S, T, hq,
                                          hkv, d, scale, ctypes.byref(st) if st else None, ds, ds0, g("dq", hq), g("dk", hkv),
                                          g("dv", hkv), wsp, size, None)


def test_bwd_refusals(lib):
    c = lambda **kw: bwd(lib, **kw)  # noqa: E731
    assert c() == HIP and c(st=state((3, 3))) == HIP and c(ds=FAKE, ds0=FAKE + (1 << 30)) == HIP
    assert c(S=0) == OK and c(off=(0, 0, 0)) == OK
    assert c(S=-1) == SHAPE and c(hq=3) == HEADS and c(off=(0, 5, 10)) == OFFSETS and c(scale=0.0) == UNSUPPORTED
    assert c(st=state((1, 8))) == PAGE and c(st=state((1, 0), heads=1)) == HEADS and c(ld=None) == NULL
    assert c(ds=FAKE + 4) == ALIGN and c(ds0=FAKE + 8) == ALIGN
    assert c(ds=FAKE, ds0=FAKE) == SHAPE and c(ds=FAKE, ds0=FAKE + 65536) == SHAPE
    for name in ("q", "k", "v", "dout", "dq", "dk", "dv"):
        assert c(**{name: t3(ptr=0)}) == NULL and c(**{name: t3(dtype=ws.WS_DTYPE_F32)}) == UNSUPPORTED
    assert c(wsp=None) == WORKSPACE and c(size=8) == WORKSPACE


def test_first_states_and_their_gradients_apart(lib):
    """Both passes run at once: dstate0 may not be written over states that dQ's reads."""
    room = 8 * 2 * 128 * 128 * 4   # the pool's bytes; dstate0's are 2 / 8 of them
    for at, rc in ((0, SHAPE), (room - 16, SHAPE), (room, HIP), (16 - room // 4, SHAPE), (-room // 4, HIP)):
        assert bwd(lib, st=state((0, 1), pool=64 * FAKE), ds0=64 * FAKE + at) == rc, at
    assert bwd(lib, ds0=FAKE) == HIP


def test_workspace_bytes(lib):
    f = lib.ws_linear_workspace_bytes
    for bad in ((0, 9, 4, 2, 128), (2, -1, 4, 2, 128), (2, 9, 0, 2, 128), (2, 9, 4, 0, 128), (2, 9, 5, 2, 128), (2, 9, 4, 2, 96)):
        assert f(*bad) == 0
    # never less for more tokens, so that a buffer for the longest batch serves every batch
    for hq, hkv, d in ((4, 2, 128), (8, 8, 64), (64, 8, 128), (600, 600, 128)):
        sizes = [f(3, t, hq, hkv, d) for t in range(0, 6000, 37)]
        assert sizes == sorted(sizes) and sizes[0] >= 3 * hkv * d * d * 4


def test_python_arguments():
    pool = torch.zeros(3, 2, 64, 64)
    for bad in (pool[:, :, :, :32], pool.double(), pool.transpose(0, 1), pool[0]):
        with pytest.raises(ValueError):
            ws.LinearState(bad, [0])
    st = ws.LinearState(pool, [2, 0])
    assert st.slots_host.dtype == torch.int32 and st.desc().num_slots == 3
    with pytest.raises(ValueError):   # not on a device
        linear._check_state(st, 2)
    with pytest.raises(ValueError):
        linear._check_state(st, 3)
    with pytest.raises(ValueError):
        linear._check_state(object(), 1)
    with pytest.raises(ValueError):
        packed._t3(torch.zeros(2, 3, 4, 5, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        packed._t3(torch.zeros(3, 4, 5, dtype=torch.float16))
    with pytest.raises(ValueError):
        packed._seq_offsets(torch.zeros(2, 2), "cpu")
