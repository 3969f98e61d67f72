"""States and f32 outputs of linear attention over many tokens of heads that forget
slowly, against 64 bits: norms within what independent roundings leave
(tests/long_decay.py), which a decay factor that is rounded each time would pass."""
import numpy as np
import pytest
import torch

import paper_2606_25041_amd as ws
from tests import gpu_support as gs
from tests import long_decay as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"


def rnd(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV).to(torch.bfloat16)


def exact(k, v, ld, s0=None):
    """The state behind the tokens k, v [n][d] (and one before them), f64."""
    n = k.shape[0]
    far = torch.arange(n - 1, -1, -1, device=DEV, dtype=torch.float64)
    S = (k.double() * torch.exp(ld * far)[:, None]).T @ v.double()
    return S if s0 is None else S + np.exp(ld * n) * s0.double()


def off(name, got, want, limit):
    err = float((got.double() - want).norm() / want.norm())
    gs.say(f"[gpu]   {name}: {err:.2e} of {limit:.2e}")
    assert err <= limit, (name, err, limit)


def pair(x):
    h = torch.tensor(x, dtype=torch.int32)
    return h, h.to(DEV)


@pytest.mark.parametrize("d,n", ((128, 32768), (64, 65536)))
def test_many_cells_join(d, n):
    """One KV head: as many cells of 64 tokens as there are, 512 or 1024 joins; the
    gradient of the first state likewise, backwards."""
    q, k, v, do = (rnd(i, n, 1, d) for i in range(4))
    scale, cells = d ** -0.5, n // 64
    limit = ref.bound(2 * cells + 2 * 8)
    for ld in (*ref.decays(64, 3), -1e-9):
        gs.say(f"[gpu] linear, {cells} cells x {d}, log decay {ld:.3e}")
        decay = torch.tensor([ld], device=DEV)
        state = ws.LinearState(torch.zeros(1, 1, d, d, device=DEV), pair([0]))
        out = ws.linear_attn_prefill(q, k, v, decay, pair([0, n]), state=state, out_dtype=torch.float32)
        want = exact(k[:, 0], v[:, 0], ld)
        off("state", state.pool[0, 0], want, limit)
        # the last token reads it (its own rounding and sum: 8 more)
        off("out", out[-1, 0], scale * (q[-1, 0].double() @ want), ref.bound(2 * cells + 2 * 8) * 2)
        ds0 = ws.linear_attn_prefill_bwd(q, k, v, do, decay, pair([0, n]), state=state, want_dstate0=True)[3]
        off("dstate0", ds0[0, 0], scale * np.exp(ld) * exact(q[:, 0].flip(0), do[:, 0].flip(0), ld), limit + 2.0 ** -22)


@pytest.mark.parametrize("d,n,heads", ((128, 16384, 512), (64, 16384, 1024)))
def test_many_chunks_of_a_cell(d, n, heads):
    """So many KV heads that a sequence is one cell: 512 chunks, of heads whose g^32
    rounds badly."""
    gs.say(f"[gpu] linear, {n // 32} chunks, {heads} heads x {d}")
    q, k, v = (rnd(i, n, 1, d).expand(n, heads, d) for i in range(3))
    lds = (ref.decays(32, 16) * (heads // 16))[:heads]
    state = ws.LinearState(torch.zeros(1, heads, d, d, device=DEV), pair([0]))
    ws.linear_attn_prefill(q, k, v, torch.tensor(lds, device=DEV), pair([0, n]), state=state)
    for h in range(0, heads, heads // 16 + 1):
        off(f"state, {lds[h]:.3e}", state.pool[0, h], exact(k[:, 0], v[:, 0], lds[h]), ref.bound(8 * n // 32))


@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("batch", (1, 64))
def test_many_steps(batch, d):
    """Token by token in place, by narrow waves and by wide ones."""
    n, heads = 4096, 8
    gs.say(f"[gpu] linear step, {batch} x {n} tokens, {heads} heads x {d}")
    q, k, v = (rnd(i, 1, n, heads, d).expand(batch, n, heads, d) for i in range(3))
    lds = ref.decays(1, heads, 1e-4, 2.0 ** -20)   # (below, f32 has too few places for S - (1 - g) S)
    state = ws.LinearState(torch.zeros(batch, heads, d, d, device=DEV), pair(list(range(batch))))
    out = torch.empty(batch, n, heads, d, device=DEV)
    ws.linear_attn_step(q, k, v, torch.tensor(lds, device=DEV), state, out=out)
    for h in range(heads):
        want = exact(k[0, :, h], v[0, :, h], lds[h])
        for b in (0, batch - 1):
            off(f"state {b}, {lds[h]:.3e}", state.pool[b, h], want, ref.bound(2 * n))
            off(f"out {b}", out[b, -1, h], d ** -0.5 * (q[0, -1, h].double() @ want), 2 * ref.bound(2 * n))
