"""Attention whose f32 output shows in how many bits the softmax weights were
held (test infrastructure only).

With scale 1 and q = (q0, 1, anything ...), a key A = 0 scores 0, a key
B = (-1, 0, ...) scores -q0 and every other key, (0, -192, 0, ...), -192, whose
weight beside A's is an exact zero (2^-277).  With v = 0 for A and v = c for B, a row that
sees nA keys A and nB keys B has
  out = nB x c / (nA + nB x),   x = exp(-q0),
so the rounding of the one weight x enters whole, with nothing to average it out.

Bound for 0 < q0 <= 2, u = 2^-24, nB <= n: scores are exact; the exponent
q0 log2 e <= 2.9 is off by 2u of itself (the constant and its product), which is
4u of x, exp2 by another 2u; weights in three bf16 parts lose 2^-8 each, u; the
sum of 3 nB products takes at most 2u an addition, 6 nB u; that of the weights
2 nB u; the quotient and its product 3u.  (10 + 8 n) u, taken as (16 + 8 n) u.
Two parts leave up to 2^-17 = 128 u.
"""
import torch

U = 2.0 ** -24
PAIRS = 2                       # pairs (A, B) of a sequence, at most
BOUND = (16 + 8 * PAIRS) * U


def queries(seed, *shape):
    """q [...][d] bf16 (CPU): q0 in [2^-5, 2], then 1, then N(0, 1)."""
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(shape, generator=g)
    q[..., 0] = 2.0 ** -5 + (2 - 2.0 ** -5) * torch.rand(shape[:-1], generator=g)
    q[..., 1] = 1
    return q.to(torch.bfloat16)


def keys(n, at, hkv, d):
    """k, v [n][hkv][d] bf16 (CPU) with pairs (A, B) at positions at, at + 1.
    Every value is one that the 4-bit cache holds."""
    k, v = torch.zeros(n, hkv, d), torch.full((n, hkv, d), 1.5)
    k[:, :, 1] = -192
    for p in at:
        k[p], v[p] = 0, 0
        k[p + 1], k[p + 1, :, 0] = 0, -1
        v[p + 1] = values(d)
    return k.to(torch.bfloat16), v.to(torch.bfloat16)


def values(d):
    c = torch.tensor([1, -1.5, 2, 3, -4, 6, .5, -1])
    return c.repeat(d // 8)


def want(q, at, lo, hi, sinks):
    """float64 [R][Hq][d] and the rows [R] that see an A and a B; lo, hi: int [R]."""
    lo, hi = torch.as_tensor(lo), torch.as_tensor(hi)

    def seen(p):
        return ((p < hi) & ((p < sinks) | (p >= lo))).double()
    zero = torch.zeros(lo.shape, dtype=torch.float64)
    na, nb = sum((seen(p) for p in at), zero), sum((seen(p + 1) for p in at), zero)
    x = torch.exp(-q[..., 0].double())
    w = nb[:, None] * x / (na[:, None] + nb[:, None] * x)
    return w[..., None] * values(q.shape[-1]).double(), (na > 0) & (nb > 0)


def in_parts(q, parts):
    """The same for one pair from weights held as a sum of bf16 values, the
    normaliser from the f32 weight (as the kernels)."""
    x = torch.exp(-q[..., 0].double()).float()
    held, left = torch.zeros_like(x, dtype=torch.float64), x.clone()
    for _ in range(parts):
        p = left.to(torch.bfloat16).float()
        held, left = held + p.double(), left - p
    return (held / (1 + x.double()))[..., None] * values(q.shape[-1]).double()


def worst(got, ref):
    """Largest error in units of the bound."""
    return float(((got.double() - ref).abs() / (BOUND * ref.abs())).max())
