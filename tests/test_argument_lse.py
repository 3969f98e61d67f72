"""An lse that the library would misread or write past is refused by the
marshalling, on the CPU (it takes a pointer to packed f32 values)."""
import types

import pytest
import torch

import paper_2606_25041_amd as ws


def test_dtype_and_layout(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    def on_device(t):   # (the shape check asks for a tensor of the current device)
        return types.SimpleNamespace(shape=t.shape, is_cuda=True, dtype=t.dtype, is_contiguous=t.is_contiguous,
                                     device=types.SimpleNamespace(index=0))
    good = torch.zeros(2, 3, 5)
    ws._check_lse(None, (2, 3, 5))
    ws._check_lse(on_device(good), (2, 3, 5))
    for bad in (good.to(torch.bfloat16), good.double(), torch.zeros(2, 5, 3).transpose(1, 2), torch.zeros(1, 3, 5).expand(2, 3, 5)):
        with pytest.raises(ValueError, match="f32"):
            ws._check_lse(on_device(bad), (2, 3, 5))
    with pytest.raises(ValueError, match="shape"):
        ws._check_lse(on_device(good), (2, 3, 4))
    with pytest.raises(ValueError, match="device"):
        ws._check_lse(good, (2, 3, 5))
