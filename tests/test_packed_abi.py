"""What the packed entry points refuse, on the CPU: every status of the C ABI
before anything is enqueued (device pointers are fake and never dereferenced), and
the Python arguments that have no meaning."""
import numpy as np
import pytest
import torch

import paper_2606_25041_amd as ws
from paper_2606_25041_amd import packed

if torch.cuda.device_count() > 0:
    pytest.skip("uses fake device pointers; CPU-only module", allow_module_level=True)

FAKE = 0x10000
OK, NULL, SHAPE, UNSUPPORTED, ALIGN, OFFSETS, PAGE, CAPACITY, HEADS, WORKSPACE, HIP = range(11)
NAMES = ("q", "k", "v", "o", "dout", "dq", "dk", "dv")


@pytest.fixture(scope="module")
def lib():
    return ws.library()


def t3(ptr=FAKE, dtype=ws.WS_DTYPE_BF16, h=4, d=128, **kw):
    s = dict(sb=0, st=h * d, sh=d)
    s.update(kw)
    return ws.Tensor4(ptr, dtype, s["sb"], s["st"], s["sh"])


def call(lib, bwd=False, off=(0, 5, 9), blocks=None, text=None, T=9, S=2, nb=None, hq=4, hkv=2, d=128, scale=0.1, lse=FAKE,
         out=None, wsp=FAKE, size=1 << 40, off_host=True, off_dev=FAKE, blocks_dev="as host", text_dev="as host", **t):
    arrays = [None if x is None else np.array(x, np.int32) for x in (off, blocks, text)]
    h = [None if x is None else x.ctypes.data for x in arrays]
    dev = lambda x, given: (None if x is None else FAKE) if given == "as host" else given  # noqa: E731
    g = lambda name: t.get(name) or t3(h=hkv if name in ("k", "v", "dk", "dv") else hq)  # noqa: E731
    ints = [h[0] if off_host else None, off_dev, h[1], dev(blocks, blocks_dev), h[2], dev(text, text_dev), S, T,
            (0 if blocks is None else len(blocks) - 1) if nb is None else nb, hq, hkv, d, scale]
    if bwd:
        return lib.ws_block_causal_prefill_packed_bwd(g("q"), g("k"), g("v"), g("o"), g("dout"), lse, *ints, g("dq"), g("dk"), g("dv"),
                                                      wsp, size, None)
    return lib.ws_block_causal_prefill_packed(g("q"), g("k"), g("v"), *ints, out or t3(h=hq), lse, None)


@pytest.mark.parametrize("bwd", (False, True))
def test_refusals(lib, bwd):
    c = lambda **kw: call(lib, bwd, **kw)  # noqa: E731
    assert c() == HIP   # valid: reaches the launch, and there is no device
    assert c(blocks=(0, 2, 5, 5, 9)) == HIP and c(blocks=(0, 5, 9), text=(0, 9)) == HIP and c(T=20) == HIP
    assert c(S=0) == OK and c(T=0) == OK and c(off=(0, 0, 0)) == OK
    assert c(S=-1) == SHAPE and c(T=-1) == SHAPE and c(nb=-1) == SHAPE and c(hq=0) == SHAPE and c(hkv=-2) == SHAPE
    assert c(T=2 ** 31 - 1) == SHAPE and (not bwd or c(T=1 << 30) == SHAPE)
    assert c(hq=5) == HEADS and c(d=80) == UNSUPPORTED
    assert c(off=(1, 5, 9)) == OFFSETS and c(off=(0, 6, 5)) == OFFSETS and c(off=(0, 5, 10)) == OFFSETS
    assert c(off_host=False) == NULL and c(off_dev=None) == NULL
    # blocks: one copy, a number without them, a bad first, order, end, a sequence inside one
    assert c(blocks=(0, 5, 9), blocks_dev=None) == NULL and c(blocks_dev=FAKE) == NULL and c(nb=2) == SHAPE
    assert c(blocks=(1, 5, 9)) == OFFSETS and c(blocks=(0, 6, 5, 9)) == OFFSETS and c(blocks=(0, 5, 8)) == OFFSETS
    assert c(blocks=(0, 4, 9)) == OFFSETS and c(blocks=(0, 9)) == OFFSETS and c(off=(0, 5, 5), blocks=(0, 4, 5)) == HIP
    assert c(text=(0, 5)) == OFFSETS and c(blocks=(0, 5, 9), text=(0, 4)) == OFFSETS and c(blocks=(0, 5, 9), text=(6, 6)) == OFFSETS
    assert c(blocks=(0, 5, 9), text=(0, 5), text_dev=None) == NULL
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert c(scale=scale) == UNSUPPORTED
    assert c(lse=FAKE + 2) == ALIGN and c(lse=None) == (NULL if bwd else HIP)
    for name in NAMES if bwd else NAMES[:3]:
        h = 2 if name in ("k", "v", "dk", "dv") else 4
        assert c(**{name: t3(ptr=0, h=h)}) == NULL and c(**{name: t3(ptr=FAKE + 8, h=h)}) == ALIGN
        assert c(**{name: t3(sh=132, h=h)}) == ALIGN and c(**{name: t3(st=-512, h=h)}) == SHAPE
        assert c(**{name: t3(dtype=ws.WS_DTYPE_F32, h=h)}) == UNSUPPORTED   # (gradients: of another dtype than the others)
    if bwd:
        f32 = {n: t3(dtype=ws.WS_DTYPE_F32, h=4 if n == "dq" else 2) for n in ("dq", "dk", "dv")}
        assert c(**f32) == HIP
        least = (8 * 4 * 9 + 255) // 256 * 256 + 8 * 9
        assert c(size=least) == HIP and c(size=least - 1) == WORKSPACE and c(wsp=None) == WORKSPACE and c(wsp=FAKE + 4) == WORKSPACE
    else:
        assert c(out=t3(dtype=ws.WS_DTYPE_F32)) == HIP and c(out=t3(ptr=0)) == NULL and c(out=t3(dtype=9)) == UNSUPPORTED
        assert c(k=t3(st=1 << 24, h=2)) == SHAPE and c(v=t3(st=1 << 24, h=2)) == SHAPE


def test_workspace_bytes(lib):
    f = lib.ws_prefill_packed_bwd_workspace_bytes
    assert f(0, 4, 2) == 0 and f(10, 4, 3) == 0 and f(10, 0, 0) == 0 and f(1 << 30, 4, 2) == 0
    sizes = [f(t, 32, 8) for t in range(1, 40000, 371)]
    assert sizes == sorted(sizes)


def test_python_arguments():
    with pytest.raises(ValueError):
        packed._blocks(None, [0], "cpu")
    with pytest.raises(ValueError):
        packed.block_causal_prefill_packed_bwd(None, None, None, None, None, None, None, grad_dtype=torch.float16)
