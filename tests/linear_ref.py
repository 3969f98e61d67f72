"""Linear attention with a decay for each head in 64 bits, token by token, and how
far the kernels may be from it.

run() is the recurrence itself:
    forwards   S <- g S + sum_j y_j z_j^T,  out = x S            (x, y, z) = (q, k, v)
    backwards  out = x (S + sum_j y_j z_j^T),  S <- g (S + ...)  from the last token on
with x [n][H][d] and y, z [n][J][H][d], J key sets summed.

How far: a product of two bf16 is exact in f32, the sums are f32.  Of a chunk of 32
tokens the scores times their weights enter the second product as two bf16 (each
half a step off at most: 2^-8 of the value, then 2^-8 of what is left: 2^-16; f32
outputs: three, 2^-24), the state that the chunk meets as one (2^-8; f32: three).
The state's sum takes values times weights in three bf16 parts.  Weights are
within 2^-20 of themselves (an exponent of up to 31 l in f32, l the logarithm of
the decay: e^-x is off by x 2^-23, and x e^-x < 1), the rest are f32 roundings, at
most 8 for each chunk that a sum passes and 64 for its own.
"""
import numpy as np
import torch

EPS = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # half a step


def run(x, y, z, log_decay, state, backwards=False):
    """f64 out [n][H][d], the state after, and three magnitudes per output:
    what the chunk's state, the scores of the last 32 tokens, and all sums amount
    to without cancelling; the same of the state."""
    x, y, z = (np.asarray(t, np.float64) for t in (x, y, z))
    n = x.shape[0]
    g = np.exp(np.asarray(log_decay, np.float64))[:, None, None]
    S = np.array(state, np.float64)
    A = np.abs(S)
    out, by_state, by_scores, every = (np.zeros((n, *x.shape[1:])) for _ in range(4))
    order = range(n - 1, -1, -1) if backwards else range(n)
    recent = []
    for t in order:
        add = np.einsum("jha,jhb->hab", y[t], z[t])
        mag = np.einsum("jha,jhb->hab", np.abs(y[t]), np.abs(z[t]))
        if not backwards:
            before = np.abs(g * S)
            S, A = g * S + add, g * A + mag
        else:
            before = np.abs(S)
            S, A = S + add, A + mag
        out[t] = np.einsum("ha,hab->hb", x[t], S)
        every[t] = np.einsum("ha,hab->hb", np.abs(x[t]), A)
        # a chunk may begin at any of the last 32 tokens: the state it met is at most
        # what is here and what has come since
        recent = [(w * g[:, :, 0], u) for w, u in recent[-31:]] + [(np.ones_like(g[:, :, 0]), t)]
        loose = sum(w * np.einsum("ha,jha,jhb->hb", np.abs(x[t]), np.abs(y[u]), np.abs(z[u])) for w, u in recent)
        by_state[t] = np.einsum("ha,hab->hb", np.abs(x[t]), before) + loose
        by_scores[t] = sum(w * np.einsum("jh,jhb->hb", np.abs(np.einsum("ha,jha->jh", x[t], y[u])), np.abs(z[u]))
                           for w, u in recent)
        if backwards:
            S, A = g * S, g * A
    return out, S, (by_state, by_scores, every), A


def chunks(n):
    return n // 32 + 2


def out_bound(out, mags, n, dtype, scale):
    by_state, by_scores, every = (m * scale for m in mags)
    slack = (8 * chunks(n) + 64) * 2.0 ** -24
    f32 = dtype == torch.float32
    return (EPS[dtype] * np.abs(out) * scale + (2.0 ** -24 if f32 else 2.0 ** -8) * by_state +
            (2.0 ** -24 if f32 else 2.0 ** -16) * by_scores + 2.0 ** -20 * by_scores + slack * every) * (1 + 2.0 ** -7) + 1e-37


def state_bound(A, n):
    return (2.0 ** -20 + (8 * chunks(n) + 64) * 2.0 ** -24) * A + 1e-37


def step_bound(out, every, n, dtype, scale):
    """The recurrent form: f32 throughout, three roundings a token and a sum of d."""
    return EPS[dtype] * np.abs(out) * scale + (4 * n + 160) * 2.0 ** -24 * every * scale + 1e-37


def forward(q, k, v, log_decay, state):
    """run() of [n][Hq][d], [n][Hkv][d]: out [n][Hq][d], the state, magnitudes."""
    hq, hkv = q.shape[1], k.shape[1]
    G = hq // hkv
    rep = lambda t: np.repeat(np.asarray(t, np.float64), G, axis=1)  # noqa: E731
    out, S, mags, A = run(q, rep(k)[:, None], rep(v)[:, None], np.repeat(np.asarray(log_decay, np.float64), G),
                          np.repeat(np.asarray(state, np.float64), G, axis=0))
    return out, S[::G], mags, A[::G]


def gradients(q, k, v, dout, log_decay, state, dstate, scale):
    """{name: (value, magnitudes or A)} of dq, dk, dv and dstate0 (without the
    output's scale in dq, dk, dv's sums)."""
    q, k, v, dout = (np.asarray(t, np.float64) for t in (q, k, v, dout))
    hq, hkv = q.shape[1], k.shape[1]
    G = hq // hkv
    rep = lambda t: np.repeat(t, G, axis=1)  # noqa: E731
    turned = np.swapaxes(np.asarray(state, np.float64), -1, -2)
    dq, _, mq, _ = run(dout, rep(v)[:, None], rep(k)[:, None], np.repeat(np.asarray(log_decay, np.float64), G),
                       np.repeat(turned, G, axis=0))
    sets = lambda t: t.reshape(t.shape[0], hkv, G, t.shape[2]).transpose(0, 2, 1, 3)  # noqa: E731
    later = np.asarray(dstate, np.float64) / scale
    dv, after, mv, A = run(k, sets(q), sets(dout), log_decay, later, True)
    dk, _, mk, _ = run(v, sets(dout), sets(q), log_decay, np.swapaxes(later, -1, -2), True)
    return {"dq": (dq, mq), "dk": (dk, mk), "dv": (dv, mv), "dstate0": (after, A)}
