"""Caches and workspaces whose memory a kernel must not be given are refused by
the marshalling, on the CPU."""
import pytest
import torch

import paper_2606_25041_amd as ws


def _caches():
    table = torch.zeros(1, 2, dtype=torch.int32)
    pool = torch.zeros(3, 2, 64, 64, dtype=torch.bfloat16)
    return ws.PagedCache(pool, pool.clone(), table), ws.PagedCache4(torch.zeros(3, 2, 68 * 64, dtype=torch.uint8), table)


def test_caches_on_the_host():
    for cache in _caches():
        with pytest.raises(ValueError, match="page table"):
            ws._check_table(cache, 1)


def test_pools(monkeypatch):
    monkeypatch.setattr(ws, "_check_pair", lambda *_: None)   # (no device copy of the table here)
    for cache in _caches():
        with pytest.raises(ValueError, match="pools"):
            ws._check_table(cache, 1)
        with pytest.raises(ValueError, match="rows"):
            ws._check_table(cache, 2)


def test_workspace():
    ws._check_workspace(None)
    with pytest.raises(ValueError, match="workspace"):
        ws._check_workspace(torch.zeros(16, dtype=torch.uint8))


def test_a_cache_with_its_own_descriptor(monkeypatch):
    """What its attributes hold is its own matter: desc() says what is read."""
    class Placed(ws.PagedCache):
        def desc(self):
            return super().desc()

    class Duck:
        page_table_host = page_table = torch.zeros(1, 2, dtype=torch.int32)

        def desc(self):
            raise AssertionError("not asked here")
    monkeypatch.setattr(ws, "_check_pair", lambda *_: None)   # (no device copy of the table here)
    pool = torch.zeros(3, 2, 64, 64, dtype=torch.bfloat16)
    ws._check_table(Placed(pool, pool, torch.zeros(1, 2, dtype=torch.int32)), 1)
    ws._check_table(Duck(), 1)
