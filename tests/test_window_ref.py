"""The float64 reference of the windowed tests, on the CPU: against a row-by-row
brute force, central differences and the textbook special cases."""
import numpy as np
import torch

from tests import window_ref as ref


def _inputs(seed, R, N, Hq, Hkv, d):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(R, Hq, d, generator=g, dtype=torch.float64), torch.randn(N, Hkv, d, generator=g, dtype=torch.float64),
            torch.randn(N, Hkv, d, generator=g, dtype=torch.float64))


def test_ranges_by_brute_force():
    """Every layout of 6 tokens in blocks with every segment start: the visible
    set of each token, from the rule in words."""
    for cuts in range(2 ** 5):
        off = [0] + [i + 1 for i in range(5) if cuts >> i & 1] + [6]
        for pick in range(3):
            starts = [min(e, s + pick * (e - s) // 2) for s, e in zip(off, off[1:])]
            for window, sinks in ((0, 0), (1, 2), (3, 1), (9, 0)):
                lo, hi = ref.ranges(off, starts, window)
                for n, (s, e) in enumerate(zip(off, off[1:])):
                    for i in range(s, e):
                        if i < starts[n]:   # an observation: the block's, and the window before the block
                            see = {j for j in range(6) if j < starts[n] and (j >= s - window or j < sinks)}
                        else:               # token-causal: up to itself, the window before itself
                            see = {j for j in range(i + 1) if j >= i - window or j < sinks}
                        assert see == {j for j in range(6) if j < hi[i] and (j < sinks or j >= lo[i])}
                        assert i in see


def test_no_window_is_plain_attention():
    q, k, v = _inputs(0, 9, 9, 4, 2, 8)
    lo, hi = ref.ranges(list(range(10)), None, 100)
    got = ref.attend(q, k, v, lo, hi, 0, 0.3)["out"][0]
    kk, vv = (x.repeat_interleave(2, 1).transpose(0, 1) for x in (k, v))
    want = torch.nn.functional.scaled_dot_product_attention(q.transpose(0, 1), kk, vv, is_causal=True, scale=0.3)
    assert (got.transpose(0, 1) - want).abs().max() < 1e-13


def test_gradients_by_differences():
    R = 11
    q, k, v = _inputs(3, R, R, 2, 1, 4)
    do = torch.randn(R, 2, 4, generator=torch.Generator().manual_seed(5), dtype=torch.float64)
    lo, hi = ref.ranges([0, 3, 3, 8, 11], [2, 3, 5, 8], 2)
    got = ref.attend(q, k, v, lo, hi, 1, 0.5, dout=do)

    def loss(*x):
        return float((ref.attend(*x, lo, hi, 1, 0.5)["out"][0] * do).sum())
    for i, name in enumerate(("dq", "dk", "dv")):
        x = [t.clone() for t in (q, k, v)]
        flat, g = x[i].view(-1), got[name][0].reshape(-1)
        for e in range(flat.numel()):
            at = float(flat[e])
            flat[e] = at + 1e-5
            up = loss(*x)
            flat[e] = at - 1e-5
            down = loss(*x)
            flat[e] = at
            assert abs((up - down) / 2e-5 - float(g[e])) < 1e-8, (name, e)


def test_keys_no_row_sees_may_hold_nan():
    q, k, v = _inputs(7, 2, 10, 2, 2, 4)
    k[3:6], v[3:6] = float("nan"), float("nan")
    got = ref.attend(q, k, v, np.array([6, 7]), np.array([9, 10]), 3, 0.5)
    assert torch.isfinite(got["out"][0]).all() and torch.isfinite(got["lse"][0]).all()
