"""The calls that the GPU tests of windows and of the 4-bit cache run reach every
kernel and kind of plan at both head dims and output types, on 256 compute
units."""
import itertools
import random

import numpy as np
import pytest

from tests import session_plan_cases as cases
from tests import session_plan_probe as probe
from tests.test_gpu_window import _layout

STEP_CLASSES = {"one split, few rows", "one split", "splits", "per stream, split", "per stream, whole"}


def test_4bit_steps():
    seen = set()
    for d, f32 in itertools.product(cases.DIMS, cases.OUTPUTS):
        for cls, hq, hkv, new, caches, lens, _ in cases.STEPS4:
            plan = probe.step4(hq, hkv, d, new, caches, lens, f32)
            assert cases.step_class(plan, hq // hkv * new) == cls and plan.f32 == f32, (plan, caches)
            assert plan.merged == (cls in ("splits", "per stream, split"))
            seen.add((cls, d, f32))
    assert len(seen) == 4 * (len(STEP_CLASSES) + 2)


def test_windowed_steps():
    seen = set()
    for d, f32 in itertools.product(cases.DIMS, cases.OUTPUTS):
        for cls, hq, hkv, new, caches, lens, _, window, sinks in cases.STEPS_WINDOW:
            plan = probe.step_window(hq, hkv, d, new, caches, lens, window, sinks, f32)
            assert cases.step_class(plan, hq // hkv * new) == cls and plan.f32 == f32, (plan, caches)
            assert plan.merged == (cls in ("splits", "per stream, split"))
            seen.add((cls, d, f32))
    assert len(seen) == 4 * len(STEP_CLASSES)


@pytest.mark.parametrize("seed", (50, 70))   # (the layouts of the prefills, and of the gradients)
@pytest.mark.parametrize("paged", (False, True))
def test_windowed_prefills(paged, seed):
    seen = set()
    for d, f32 in itertools.product(cases.DIMS, cases.OUTPUTS):
        for groups, B, hq, hkv, L, blocks, text, window, sinks in cases.PREFILLS:
            lay = [_layout(seed + 100 * b, L, blocks, text) for b in range(B)]
            off = np.concatenate([x[0] for x in lay])
            starts = np.concatenate([x[1] for x in lay]) if text else None
            assert probe.prefill_window(hq, hkv, d, off, starts, window, sinks, paged, f32) == groups
            seen.add((groups, d, f32))
    assert len(seen) == 8


def test_windowed_steps_stay_in_the_workspace():
    g = random.Random(11)
    seen = set()
    for cus in (256, 304, 32, 1):
        for _ in range(300):
            hkv, G, new = g.choice((1, 2, 3, 8, 24, 64, 300)), g.choice((1, 3, 4, 8, 16)), g.choice((1, 1, 2, 3, 17, 128, 512))
            b, d, f32 = g.choice((1, 1, 2, 4, 31, 32, 33)), g.choice((64, 128)), g.random() < .5
            caches = [g.choice((0, 1, 63, 64, 65, int(np.exp(g.uniform(0, 12))))) for _ in range(b)]
            lens = [g.randint(1, new) for _ in range(b)] if g.random() < .5 else None
            window, sinks = (g.choice((0, 1, int(np.exp(g.uniform(0, 12))), 2 ** 31 - 1)) for _ in range(2))
            args = (hkv * G, hkv, d, new, caches, lens, window, sinks, f32, cus)
            rc, used, need, plan = probe.step_window_workspace(*args)
            assert rc == 0 and used <= need, args
            seen.add((plan[0], plan[1] > 1))
            if need:
                assert probe.step_window_workspace(*args, given=need - 1)[0] == 9
    assert seen == {(False, False), (False, True), (True, False), (True, True)}


def test_4bit_steps_of_blocks_of_different_lengths_stay_in_the_workspace():
    g = random.Random(12)
    seen = set()
    for cus in (256, 304, 32, 1):
        for _ in range(300):
            hkv, G, new = g.choice((1, 2, 3, 8, 24, 64, 300)), g.choice((1, 3, 4, 8, 16)), g.choice((1, 2, 3, 17, 128, 512))
            b, d, f32 = g.choice((1, 1, 2, 4, 31, 32, 33)), g.choice((64, 128)), g.random() < .5
            caches = [g.choice((0, 1, 63, 64, 65, int(np.exp(g.uniform(0, 12))))) for _ in range(b)]
            args = (hkv * G, hkv, d, new, caches, [g.randint(1, new) for _ in range(b)], f32, cus)
            rc, used, need, plan = probe.step4_workspace(*args)
            assert rc == 0 and used <= need, args
            seen.add(plan)
            if need:
                assert probe.step4_workspace(*args, given=need - 1)[0] == 9
    assert seen == {(True, False), (False, True), (False, False)}
