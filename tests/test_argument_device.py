"""Tensors of another device than the current one, whose stream and code object a
call would launch, are refused by the marshalling, on the CPU."""
import types

import pytest
import torch

import paper_2606_25041_amd as ws


def on(index):
    t = torch.zeros(2, dtype=torch.int32)
    return types.SimpleNamespace(shape=t.shape, is_cuda=True, device=types.SimpleNamespace(index=index, type="cuda"),
                                 dtype=t.dtype, is_contiguous=t.is_contiguous, element_size=lambda: 2)


def test_tensors_of_another_device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    host = torch.zeros(2, dtype=torch.int32)
    ws._shape("q", on(1), (2,))
    ws._check_pair("lens", host, on(1))
    ws._check_workspace(on(1))
    for call in (lambda: ws._shape("q", on(0), (2,)), lambda: ws._check_pair("lens", host, on(0)),
                 lambda: ws._check_workspace(on(0))):
        with pytest.raises(ValueError, match="current device"):
            call()
    cache = types.SimpleNamespace(page_table_host=host, page_table=on(1), k_pool=on(1), v_pool=on(0))
    with pytest.raises(ValueError, match="current device"):
        ws._check_table(cache, 1)
    cache.v_pool = on(1)
    ws._check_table(cache, 1)
