"""The construction of tests/f32_weights.py on the CPU: its closed form against
attention in float64, and its bound, which weights in three bf16 parts keep and
weights in two do not, on every call that the GPU test makes."""
import torch

from tests import f32_weights as fw
from tests import session_plan_cases as cases
from tests import window_ref


def test_closed_form():
    n, hkv, d, sinks, window = 300, 2, 64, 3, 100
    at = [0, 150]
    k, v = fw.keys(n, at, hkv, d)
    q = fw.queries(1, n, 4, d)
    lo, hi = window_ref.ranges([0, 2, 90, 200, n], [2, 50, 200, 210], window)
    ref, rows = fw.want(q, at, lo, hi, sinks)
    got = window_ref.attend(q, k, v, lo, hi, sinks, 1.0)["out"][0]
    assert rows.sum() > 200
    assert (got[rows] - ref[rows]).abs().max() < 1e-13


def test_two_parts_do_not_pass():
    sizes = [(len(c[4]), c[3], c[1], d) for c in cases.STEPS4 + cases.STEPS_WINDOW for d in cases.DIMS]
    sizes += [(c[1], c[4], c[2], d) for c in cases.PREFILLS for d in cases.DIMS]
    for B, L, H, d in sizes:
        q = fw.queries(B * L + H, B, L, H, d)
        x = torch.exp(-q[..., 0].double())
        ref = (x / (1 + x))[..., None] * fw.values(d).double()
        assert fw.worst(fw.in_parts(q, 3), ref) < 0.2
        assert fw.worst(fw.in_parts(q, 2), ref) > 1.5, (B, L, H, d)
