"""The 4-bit reference on the CPU: hand-worked blocks, idempotence, the error
bound that include/ws_attn.h states, and the format of the benchmark's inputs."""
import numpy as np
import torch

from perf import operators
from tests import cache4_ref as ref


def _block(*x):
    return torch.tensor(list(x) + [0.0] * (32 - len(x))).to(torch.bfloat16)


def test_hand_worked():
    codes, scales = ref.encode(_block(6, 5, 2.5, 1.75, 0.25, 0.75, -3.5, -0.2))
    assert scales[0] == 127   # amax 6: scale 1
    assert codes[:8].tolist() == [7, 6, 4, 4, 0, 2, 14, 8]   # 5 -> 4, 2.5 -> 2, 1.75 -> 2, 0.25 -> 0, 0.75 -> 1, -3.5 -> -4
    codes, scales = ref.encode(_block(6.03125, 1))
    assert scales[0] == 128 and codes[0] == 5   # scale 2: 3.015625 -> 3
    assert ref.encode(_block(0))[1][0] == 27    # all zero: 2^-100
    assert ref.encode(_block(3.38e38))[1][0] == 252 and ref.rounded(_block(3.38e38))[0] == 6 * 2.0 ** 125
    assert ref.rounded(_block(1.0, float("inf"))).isnan().all() and ref.encode(_block(float("nan")))[1][0] == 255


def test_idempotent_and_bounded():
    g = torch.Generator().manual_seed(1)
    x = (torch.randn(4096, 64, generator=g) * torch.exp2(torch.randint(-90, 100, (4096, 1), generator=g))).to(torch.bfloat16)
    y = ref.rounded(x)
    assert torch.equal(ref.rounded(y), y)
    scale = torch.from_numpy(2.0 ** (ref.encode(x)[1].astype(np.float64) - 127)).repeat_interleave(32, -1)
    err = (x.double() - y.double()).abs()
    assert (err <= torch.maximum(scale / 4, x.double().abs() / 5)).all()
    top = x.double().abs().reshape(4096, 2, 32).amax(-1).repeat_interleave(32, -1)
    assert (err <= top / 5).all()


def test_benchmark_inputs_have_this_format():
    g = torch.Generator().manual_seed(2)
    x = (torch.randn(999, 3, 128, generator=g) * 3).to(torch.bfloat16)
    want = ref.decode(*ref.encode(x))
    assert np.array_equal(operators._values(*operators._quantise(x)).numpy(), want)
    assert np.array_equal(operators._rounded4(x).numpy(), want)
