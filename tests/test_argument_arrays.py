"""Host and device int32 arrays that the library would misread are refused by the
marshalling, on the CPU: strided ones (it reads packed arrays), both copies on
one side (a kernel would read host memory, or the host device memory)."""
import pytest
import torch

import paper_2606_25041_amd as ws


def ints(n):
    return torch.arange(n, dtype=torch.int32)


def test_lengths():
    with pytest.raises(ValueError, match="pair"):
        ws._check_lens(ints(2), ints(2), 2)   # no device copy
    with pytest.raises(ValueError, match="contiguous"):
        ws._check_lens(ints(4)[::2], ints(2), 2)
    with pytest.raises(ValueError, match="contiguous"):
        ws._check_lens(ints(2), ints(4)[::2], 2)
    with pytest.raises(ValueError, match="contiguous"):
        ws._check_lens(ints(1).expand(2), ints(2), 2)


def test_starts():
    with pytest.raises(ValueError, match="pair"):
        ws._int32_pair((ints(2), ints(2)), (2,), "cpu")
    with pytest.raises(ValueError, match="contiguous"):
        ws._int32_pair((ints(1).expand(2), ints(2)), (2,), "cpu")
    with pytest.raises(ValueError, match="contiguous"):
        ws._int32_pair((ints(2).long(), ints(2)), (2,), "cpu")


def test_block_offsets():
    off = torch.tensor([[0, 4]], dtype=torch.int32)
    for host, dev, match in ((off, off, "pair"), (off.to("meta"), off, "pair"), (off.long(), off, "contiguous"),
                             (off, off.long(), "contiguous"), (ints(4)[None, ::2], off, "contiguous"),
                             (off, ints(4)[None, ::2], "contiguous")):
        with pytest.raises(ValueError, match=match):
            ws._check_offsets(host, dev, 1, 1)
    with pytest.raises(ValueError, match="num_blocks"):
        ws._check_offsets(off, off, 2, 1)
    assert ws._offsets([[0, 3, 5]], "cpu")[2] == 2
