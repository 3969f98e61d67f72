"""The reference of linear attention (tests/linear_ref.py) against the sum over all
earlier tokens written out, its gradients against differences."""
import numpy as np
import pytest

from tests import linear_ref as ref


def case(seed, n, hq, hkv, d):
    r = np.random.default_rng(seed)
    draw = lambda *s: r.standard_normal(s)  # noqa: E731
    return draw(n, hq, d), draw(n, hkv, d), draw(n, hkv, d), -r.random(hkv), draw(hkv, d, d)


def plain(q, k, v, ld, s0):
    n, hq, d = q.shape
    G = hq // k.shape[1]
    out = np.zeros_like(q)
    for h in range(hq):
        g = np.exp(ld[h // G])
        for i in range(n):
            for j in range(i + 1):
                out[i, h] += g ** (i - j) * (q[i, h] @ k[j, h // G]) * v[j, h // G]
            out[i, h] += g ** (i + 1) * (q[i, h] @ s0[h // G])
    last = np.stack([np.exp(ld[h] * n) * s0[h] + sum(np.exp(ld[h] * (n - 1 - j)) * np.outer(k[j, h], v[j, h]) for j in range(n))
                     for h in range(k.shape[1])])
    return out, last


@pytest.mark.parametrize("hq,hkv", ((2, 2), (4, 2), (3, 1)))
def test_recurrence_is_the_sum(hq, hkv):
    q, k, v, ld, s0 = case(1, 7, hq, hkv, 3)
    out, last = plain(q, k, v, ld, s0)
    got, S, mags, A = ref.forward(q, k, v, ld, s0)
    assert np.allclose(got, out, rtol=0, atol=1e-12) and np.allclose(S, last, rtol=0, atol=1e-12)
    assert all((m >= 0).all() for m in mags) and (A >= np.abs(S) - 1e-12).all()
    assert (mags[2] >= np.abs(out) - 1e-12).all()


def test_gradients_against_differences():
    q, k, v, ld, s0 = case(2, 6, 4, 2, 3)
    r = np.random.default_rng(3)
    do, ds, scale, eps = r.standard_normal(q.shape), r.standard_normal(s0.shape), 0.7, 1e-6
    got = ref.gradients(q, k, v, do, ld, s0, ds, scale)

    def loss(q, k, v, s0):
        out, last = plain(q, k, v, ld, s0)
        return scale * (out * do).sum() + (last * ds).sum()
    for name, i in (("dq", 0), ("dk", 1), ("dv", 2), ("dstate0", 3)):
        args = [q, k, v, s0]
        for at in np.ndindex(*args[i].shape):
            up, down = [a.copy() for a in args], [a.copy() for a in args]
            up[i][at] += eps
            down[i][at] -= eps
            assert abs((loss(*up) - loss(*down)) / (2 * eps) - scale * got[name][0][at]) < 1e-6, (name, at)


@pytest.mark.parametrize("wrong", ("decay", "order", "state", "heads"))
def test_mistakes_are_out_of_bounds(wrong):
    """Planted in the oracle: the bound of a bf16 output tells them."""
    import torch
    q, k, v, ld, s0 = case(4, 70, 4, 2, 64)
    ld = ld / 30
    out, S, mags, A = ref.forward(q, k, v, ld, s0)
    if wrong == "decay":
        bad, T, _, _ = ref.forward(q, k, v, ld * 1.5, s0)
    elif wrong == "order":   # a token that does not see itself
        bad, T, _, _ = ref.forward(q, np.concatenate((k[:1] * 0, k[:-1])), np.concatenate((v[:1] * 0, v[:-1])), ld, s0)
    elif wrong == "state":
        bad, T, _, _ = ref.forward(q, k, v, ld, np.swapaxes(s0, -1, -2))
    else:
        bad, T, _, _ = ref.forward(q[:, ::-1], k, v, ld, s0)
    assert (np.abs(bad - out) > ref.out_bound(out, mags, 70, torch.bfloat16, 1.0)).any()
    if wrong != "heads":
        assert (np.abs(T - S) > ref.state_bound(A, 70)).any()
