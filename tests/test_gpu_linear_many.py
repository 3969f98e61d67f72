"""A linear prefill of more than 2^20 sequences whose states go through the workspace:
every launch of it holds them all."""
import pytest
import torch

import paper_2606_25041_amd as ws
from tests import gpu_support as gs

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_a_million_states():
    """Sequences of one token behind a long one, 64 KiB of state each: S' = g S + k v^T,
    a product and two roundings of f32 (2^-23 of the sum of the magnitudes)."""
    d, count, long = 128, (1 << 20) + 3, 5000
    need = 2 * (count + 1) * d * d * 4
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < need + (8 << 30):
        pytest.skip(f"needs {need >> 30} GiB of device memory")
    gs.say(f"[gpu] linear prefill, {count} sequences")
    T = long + count
    g = torch.Generator(DEV).manual_seed(1)
    q, k, v = (torch.randn(T, 1, d, generator=g, device=DEV).to(torch.bfloat16) for _ in range(3))
    off = torch.cat((torch.zeros(1, dtype=torch.int32), torch.arange(long, T + 1, dtype=torch.int32)))
    slots = torch.arange(count + 1, dtype=torch.int32).flip(0).contiguous()
    pool = torch.full((count + 1, 1, d, d), 0.5, device=DEV)
    decay = torch.tensor([-0.25], device=DEV)
    state = ws.LinearState(pool, (slots, slots.to(DEV)))
    ws.linear_attn_prefill(q, k, v, decay, (off, off.to(DEV)), state=state)
    torch.cuda.synchronize()
    for s in (1, 2, 65536, 1 << 19, count - 1, count):
        a = long + s - 1
        kept, new = 0.5 * torch.exp(decay.double()), k[a, 0].double()[:, None] * v[a, 0].double()
        got = pool[int(slots[s]), 0].double()
        # (g itself is within 2^-23)
        assert ((got - kept - new).abs() <= 2.0 ** -22 * (kept + new.abs())).all(), s
    del pool, state
    torch.cuda.empty_cache()
