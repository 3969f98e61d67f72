"""The bounds of tests/long_decay.py tell a rounded decay factor, and a decay that is
rounded by itself, from S + ((g^n - 1) S + x)."""
import numpy as np
import pytest

from tests import long_decay as ref


@pytest.mark.parametrize("n,steps", ((64, 512), (64, 1024), (32, 1024), (1, 4096)))
def test_a_rounded_factor_is_out_of_bounds(n, steps):
    x = np.random.default_rng(steps).standard_normal((steps, 4096)).astype(np.float32)
    for ld in ref.decays(n, 3):
        assert ref.off(n, ld) > 0.9 * 2.0 ** -25
        limit = ref.bound(2 * steps)
        assert ref.error(*ref.recurrence(x, ld, n, "factor")) > limit
        assert ref.error(*ref.recurrence(x, ld, n, "once")) <= limit


def test_a_decay_rounded_by_itself_is_out_of_bounds():
    """One unit of the last place a join of 64 tokens."""
    x = np.random.default_rng(1).standard_normal((1024, 4096)).astype(np.float32)
    assert ref.error(*ref.recurrence(x, -1e-9, 64, "twice")) > ref.bound(2 * 1024)
    assert ref.error(*ref.recurrence(x, -1e-9, 64, "once")) <= ref.bound(2 * 1024)


def test_steps_of_products_of_bf16():
    """Token by token the decay is rounded by itself: from 2^-20 a token on within the
    bound, a rounded factor is not."""
    import torch
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(4096, 64, generator=g).to(torch.bfloat16).float().numpy() for _ in range(2))
    x = (k[:, :, None] * v[:, None, :]).reshape(4096, -1)
    for ld in ref.decays(1, 3, 1e-4, 2.0 ** -20):
        assert ref.error(*ref.recurrence(x, ld, 1, "factor")) > ref.bound(2 * 4096)
        assert ref.error(*ref.recurrence(x, ld, 1, "twice")) <= ref.bound(2 * 4096)
