"""Windowed calls and steps over a 4-bit cache through every kernel and kind of
plan (tests/session_plan_cases.py) at both head dims and output types: the checks
of tests/test_gpu_cache4.py and tests/test_gpu_window.py, every element within
its derived bound, on these calls."""
import pytest
import torch

from tests import gpu_support as gs
from tests import session_plan_cases as cases
from tests import test_gpu_cache4 as cache4
from tests import test_gpu_window as windows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("f32", cases.OUTPUTS)
@pytest.mark.parametrize("d", cases.DIMS)
@pytest.mark.parametrize("case", range(len(cases.STEPS4)))
def test_4bit_step(case, d, f32, monkeypatch):
    cls, hq, hkv, new, caches, lens, starts = cases.STEPS4[case]
    gs.say(f"[gpu] 4-bit step, {cls}")
    monkeypatch.setattr(cache4, "STEPS", [(hq, hkv, d, new, caches, lens, starts, f32)])
    cache4.test_step(0)


@pytest.mark.parametrize("f32", cases.OUTPUTS)
@pytest.mark.parametrize("d", cases.DIMS)
@pytest.mark.parametrize("case", range(len(cases.STEPS_WINDOW)))
def test_windowed_step(case, d, f32, monkeypatch):
    cls, hq, hkv, new, caches, lens, starts, window, sinks = cases.STEPS_WINDOW[case]
    gs.say(f"[gpu] windowed step, {cls}")
    monkeypatch.setattr(windows, "STEPS", [(hq, hkv, d, new, caches, lens, starts, window, sinks, f32)])
    windows.test_step(0)


@pytest.mark.parametrize("f32", cases.OUTPUTS)
@pytest.mark.parametrize("d", cases.DIMS)
@pytest.mark.parametrize("paged", (False, True))
@pytest.mark.parametrize("case", range(len(cases.PREFILLS)))
def test_windowed_prefill(case, paged, d, f32, monkeypatch):
    groups, B, hq, hkv, L, blocks, text, window, sinks = cases.PREFILLS[case]
    gs.say(f"[gpu] windowed prefill, {groups} key groups")
    monkeypatch.setattr(windows, "PREFILLS", [(B, hq, hkv, d, L, blocks, text, window, sinks, paged, f32)])
    windows.test_prefill(0)


@pytest.mark.parametrize("d", cases.DIMS)
def test_gradients_behind_a_forward_of_256_row_tiles(d, monkeypatch):
    groups, B, hq, hkv, L, blocks, text, window, sinks = cases.PREFILLS[0]
    assert groups == 1
    monkeypatch.setattr(windows, "GRADS", [(B, hq, hkv, d, L, blocks, text, window, sinks, d == 128)])
    windows.test_gradients(0, "full")
    torch.cuda.synchronize()
