"""How far sums that decay slowly may be off after many steps, and decays whose
rounded factors would show.

A state S <- g S + x in f32, N roundings to nearest in all that its whole size goes
through: each is off by at most 2^-24 of the value, evenly spread, so 2^-24 / sqrt(3)
in the root mean square, and they do not depend on each other: N of them
2^-24 sqrt(N / 3) of the norm.  Twice that is allowed here, and 2^-23 + 2^-24 for the
weights of a chunk's tokens (each of 32 within 2^-23, hardware exp2) and their split
into three bf16.  A factor g^n that is itself rounded is off the same way each time:
by up to 2^-25 below 1, and a term that is passed on a times by a of that; of N equal,
uncorrelated ones the norm is off by 2^-25 N / sqrt(3), which is more from a hundred
steps on.
"""
import numpy as np


def bound(roundings):
    return 2.0 ** -23 + 2.0 ** -24 + 2 * 2.0 ** -24 * np.sqrt(roundings / 3.0)


def off(n, ld):
    """The relative error of g^n rounded to f32 (ld an f32 value)."""
    x = np.float64(n) * np.float64(np.float32(ld))
    return abs(np.float64(np.float32(np.exp(x))) / np.exp(x) - 1)


def decays(n, count, fastest=1e-5, slowest=1e-7):
    """f32 log decays between them for which g^n is a near worst case of its rounding."""
    ld = -np.float32(np.geomspace(slowest, fastest, 400 * count))
    out = []
    for part in np.array_split(ld, count):
        out.append(max(part.tolist(), key=lambda x: off(n, x)))
    return out


def recurrence(x, ld, n, kind):
    """S <- g^n S + x_i in f32 over i, and in f64.  kind: "factor", g^n rounded;
    "twice", S + (g^n - 1) S rounded before x_i is added (each time the same way where
    that is few units of S's last place); "once", S + ((g^n - 1) S + x_i)."""
    e = np.float64(n) * np.float64(np.float32(ld))
    g, less = np.float32(np.exp(e)), np.float32(np.expm1(e))
    f32 = lambda t: t.astype(np.float32)  # noqa: E731
    S, exact = np.zeros_like(x[0]), np.zeros(x[0].shape)
    for t in x:
        wide = S.astype(np.float64)
        S = f32(g * S + t) if kind == "factor" else f32(f32(wide + less * wide) + t) if kind == "twice" else f32(S + f32(less * wide + t))
        exact = np.exp(e) * exact + t.astype(np.float64)
    return S, exact


def error(got, want):
    return float(np.linalg.norm(np.asarray(got, np.float64) - want) / np.linalg.norm(want))
