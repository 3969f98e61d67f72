"""Windowed attention and its gradients from their definition in float64, with
the error bounds of kernels that round where the HIP kernels do (test
infrastructure only).

A bf16 rounding is off by at most 2^-8 of the value, a f32 one by 2^-24.
With A = sum_j p_j |v_j| and T = max_j scale sum |q_d k_jd|:
  score     off by  es = (d + 8) 2^-24 T, so a weight by a factor 1 + 3 es
            (its exponent and the normaliser's, and exp2 and log2 themselves)
  out bf16  weights and output in bf16, (a step in splits) partials in f16 under
            a power of two per row that puts the row's largest past 2^14: a
            partial is off by 2^-11 of itself or, as a subnormal (steps of
            2^-24), by 2^-25, so 2^-39 of the row's largest:
            3 * 2^-8 A + 2^-39 max_d A
  out f32   weights as two bf16 values: 2^-16 A; f32 sums over n keys:
            2^-24 (64 + sqrt n) A
  lse       es + 2^-20 (1 + |lse|)
Gradients, with D = <dO, O> from the bf16 output (out's bound e_o):
  eD  = sum_d |dO_d| e_o,d,   |dS| off by  eS = P (eD + 2^-14 (|dP| + |D|)) + 2^-8 |dS|
  dV  2^-8 sum_i P |dO|;   dQ scale sum_j eS |k|;   dK scale sum_i eS |q|
and 2^-8 of the value where it is stored as bf16.  Each bound is doubled for
the second-order terms and f32 sums it leaves out.
"""
import numpy as np
import torch

H = 2.0 ** -8


def ranges(offsets, starts, window):
    """(anchor - window, key end) of every token of one sequence, from block
    offsets [nb + 1] and segment starts [nb] (or None)."""
    lo, hi = [], []
    for n in range(len(offsets) - 1):
        s, e = int(offsets[n]), int(offsets[n + 1])
        tau = e if starts is None else int(starts[n])
        for i in range(s, e):
            lo.append((i if i >= tau else s) - window)
            hi.append(max(tau, i + 1))
    return np.asarray(lo, np.int64), np.asarray(hi, np.int64)


def step_ranges(cached, new, start, window):
    """The same for a step's new tokens (start None: no segment)."""
    lo, hi = ranges([0, new], None if start is None else [min(start, new)], window)
    return lo + cached, hi + cached


def attend(q, k, v, lo, hi, sinks, scale, dout=None, f32=False):
    """q [R][Hq][d], k, v [N][Hkv][d] (any float type, one device).  Returns a
    dict name -> (float64 value, bound) for out [R][Hq][d], lse [Hq][R] and,
    given dout, dq, dk, dv as f32 (``bf16_bound`` adds the rounding).
    Keys that no row sees may hold anything."""
    R, Hq, d = q.shape
    N, Hkv = k.shape[:2]
    G = Hq // Hkv
    dev = q.device
    lo, hi = torch.as_tensor(lo, device=dev), torch.as_tensor(hi, device=dev)
    j = torch.arange(N, device=dev)
    see = (j[None] < hi[:, None]) & ((j[None] < sinks) | (j[None] >= lo[:, None]))
    used = see.any(0)
    kz = torch.where(used[:, None, None], k.double(), 0.0)
    vz = torch.where(used[:, None, None], v.double(), 0.0)
    res = {n: (torch.zeros(s, dtype=torch.float64, device=dev), torch.zeros(s, dtype=torch.float64, device=dev))
           for n, s in (("out", (R, Hq, d)), ("lse", (Hq, R)), ("dq", (R, Hq, d)), ("dk", (N, Hkv, d)),
                        ("dv", (N, Hkv, d)))}
    for h in range(Hq):
        K, V, Q = kz[:, h // G], vz[:, h // G], q[:, h].double()
        s = torch.where(see, scale * (Q @ K.t().contiguous()), -torch.inf)
        lse = torch.logsumexp(s, 1)
        p = torch.exp(s - lse[:, None])
        T = (scale * (Q.abs() @ K.abs().t().contiguous()) * see).amax(1)
        es = (d + 8) * 2.0 ** -24 * T
        o, A = p @ V, p @ V.abs()
        rows = 0.0 if f32 else 2.0 ** -39 * A.amax(1, keepdim=True)
        e = rows + A * ((2.0 ** -16 + 2.0 ** -24 * (64 + N ** 0.5) if f32 else 3 * H) + 3 * es[:, None])
        res["out"][0][:, h], res["out"][1][:, h] = o, 2 * e
        res["lse"][0][h], res["lse"][1][h] = lse, 2 * (es + 2.0 ** -20 * (1 + lse.abs()))
        if dout is None:
            continue
        dO = dout[:, h].double()
        dP, D = dO @ V.t().contiguous(), (dO * o).sum(1, keepdim=True)
        dS = p * (dP - D)
        eD = (dO.abs() * 3 * H * A).sum(1, keepdim=True)
        eS = p * (eD + 2.0 ** -14 * (dP.abs() + D.abs())) + (H + 3 * es[:, None]) * dS.abs()
        c = lambda x: x.t().contiguous()  # noqa: E731
        for name, at, x, y in (("dq", (slice(None), h), scale * (dS @ K), scale * (eS @ K.abs())),
                               ("dk", (slice(None), h // G), scale * (c(dS) @ Q), scale * (c(eS) @ Q.abs())),
                               ("dv", (slice(None), h // G), c(p) @ dO, (H + 2.0 ** -14) * (c(p) @ dO.abs()))):
            res[name][0][at] += x
            res[name][1][at] += 2 * y
    return res if dout is not None else {n: res[n] for n in ("out", "lse")}


def check(name, got, want, bf16=False):
    """Every element of got within its bound (and what is stored as bf16 by one
    more rounding)."""
    ref, tol = want
    err = (got.double() - ref).abs()
    tol = tol + (H * (ref.abs() + tol) if bf16 else 0) + 1e-30
    worst = float((err / tol).max()) if err.numel() else 0.0
    assert worst <= 1, (name, worst, float(err.max()))   # (NaN fails too)
