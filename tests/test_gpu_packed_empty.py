"""Sequences without tokens, and blocks without, in any number between others: a packed
call's outputs and gradients are those of the batch without them, bit for bit."""
import numpy as np
import pytest
import torch

import paper_2606_25041_amd as ws
from tests import gpu_support as gs

pytestmark = pytest.mark.gpu
DEV = "cuda"


def pair(x):
    h = torch.as_tensor(np.asarray(x), dtype=torch.int32).contiguous()
    return h, h.to(DEV)


def spread(cuts, empty):
    """The offsets with empty[i] more of cut i."""
    return np.repeat(cuts, 1 + np.asarray(empty))


@pytest.mark.parametrize("form", ("causal", "blocks", "segments"))
@pytest.mark.parametrize("lens,empty", (
    ([10, 10], [0, 1000, 0]), ([10, 10], [0, 63, 0]), ([10, 10], [0, 64, 0]), ([10, 10], [70, 65, 3]),
    ([1] * 40, [100] * 41), ([300, 5, 40], [0, 5000, 130, 9]), ([3, 1, 2] * 30, [0, 1, 70] * 30 + [200])))
def test_empty_ones_change_nothing(lens, empty, form):
    gs.say(f"[gpu] packed, {sum(empty)} empty sequences between {len(lens)}, {form}")
    hq, hkv, d = 4, 2, 64
    g = torch.Generator(DEV).manual_seed(1)
    cuts = np.concatenate(([0], np.cumsum(lens)))
    T = int(cuts[-1])
    q, k, v, do = (torch.randn(T, h, d, generator=g, device=DEV).to(torch.bfloat16) for h in (hq, hkv, hkv, hq))
    # blocks: a cut in the middle of every sequence too
    edges = np.unique(np.concatenate((cuts, (cuts[:-1] + cuts[1:]) // 2)))
    at = np.isin(edges, cuts)
    more = np.zeros(len(edges), int)
    more[at] = empty

    def run(seqs, blocks):
        kw = {}
        if form != "causal":
            kw["block_offsets"] = pair(blocks)
            if form == "segments":
                kw["text_starts"] = pair((blocks[:-1] + blocks[1:]) // 2)
        out, lse = ws.block_causal_prefill_packed(q, k, v, pair(seqs), want_lse=True, **kw)
        return [out, lse, *ws.block_causal_prefill_packed_bwd(q, k, v, out, do, lse, pair(seqs), **kw)]

    for a, b in zip(run(cuts, edges), run(spread(cuts, empty), spread(edges, more))):
        assert torch.equal(a, b)
