"""The 4-bit cache format in numpy (test infrastructure only): blocks of 32 along
the last axis, rounded by comparing distances in float64."""
import numpy as np
import torch

VALUES = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
EVEN_FIRST = (0, 2, 4, 6, 1, 3, 5, 7)   # a tie keeps the even code


def encode(x):
    """Codes [...][d] (0..15) and scale bytes [...][d / 32] of a bf16 CPU tensor."""
    y = x.double().numpy().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = np.abs(y).max(-1, keepdims=True)
    bad = ~np.isfinite(top)
    top = np.where(bad, 0, top)
    e = np.full(top.shape, -100)
    for _ in range(225):
        e = np.where((top > 6 * 2.0 ** e) & (e < 125), e + 1, e)
    a = np.abs(np.where(bad, 0, y)) / 2.0 ** e
    code, dist = np.zeros(a.shape, np.int64), np.full(a.shape, np.inf)
    for c in EVEN_FIRST:
        near = np.abs(a - VALUES[c])
        code, dist = np.where(near < dist, c, code), np.minimum(near, dist)
    code = code + 8 * np.signbit(y)
    return code.reshape(x.shape), np.where(bad, 254 + 1, e + 127)[..., 0].astype(np.uint8)


def decode(codes, scales):
    """float64 values of codes [...][d] and scale bytes [...][d / 32]."""
    v = np.where(codes >= 8, -1.0, 1.0) * VALUES[codes & 7]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, 32, -1)


def rounded(x):
    """A bf16 tensor as the cache returns it (bf16, same device)."""
    return torch.from_numpy(decode(*encode(x.cpu()))).to(torch.bfloat16).to(x.device)
