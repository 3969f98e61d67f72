"""Linear attention with a decay for each head (include/ws_attn.h states it).

Token i of a sequence, with g = exp(log_decay) of its KV head:
    S_i = g S_(i-1) + k_i v_i^T,    o_i = scale * q_i S_i.
As the rest of the package this is marshalling only; the native module takes
the common case, the ctypes code here the others, with the checks and errors.

  LinearState(pool, slots): sessions' states
  linear_attn_prefill(q, k, v, log_decay, seq_offsets, ...): packed sequences, chunked
  linear_attn_prefill_bwd(q, k, v, dout, log_decay, seq_offsets, ...): its gradients
  linear_attn_step(q, k, v, log_decay, state, ...): a few new tokens
  linear_workspace_bytes(num_seqs, total_tokens, num_q_heads, num_kv_heads, head_dim)
"""
import ctypes
import math

import torch

from . import (Tensor4, _check, _check_pair, _here, _int32_pair, _native, _ptr, _shape, _stream, _t4, library)
from .packed import _seq_offsets, _t3, _workspace

WS_STATE_RESET, WS_STATE_KEEP = 1, 2


class LinearStateDesc(ctypes.Structure):
    _fields_ = [("pool", ctypes.c_void_p), ("slots_dev", ctypes.c_void_p), ("slots_host", ctypes.c_void_p),
                ("num_slots", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


def declare(lib):
    """Argument types of the linear entry points."""
    P, I32, F, N = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t
    T, ST = Tensor4, ctypes.POINTER(LinearStateDesc)
    lib.ws_linear_attn_prefill.restype = ctypes.c_int
    lib.ws_linear_attn_prefill.argtypes = [T, T, T, P, P, P, I32, I32, I32, I32, I32, F, ST, I32, T, P, N, P]
    lib.ws_linear_attn_step.restype = ctypes.c_int
    lib.ws_linear_attn_step.argtypes = [T, T, T, P, ST, P, P, I32, I32, I32, F, I32, T, P]
    lib.ws_linear_attn_prefill_bwd.restype = ctypes.c_int
    lib.ws_linear_attn_prefill_bwd.argtypes = [T, T, T, T, P, P, P, I32, I32, I32, I32, I32, F, ST, P, P, T, T, T, P, N, P]
    lib.ws_linear_workspace_bytes.restype = N
    lib.ws_linear_workspace_bytes.argtypes = [I32, I32, I32, I32, I32]


class LinearState:
    """Caller-owned states of sessions' linear attention.

    pool: f32 device [num_slots][num_kv_heads][head_dim][head_dim], contiguous;
    slots: int32 [batch], the slot of each session of a call (array-like, or a
    (host, device) pair).
    """

    def __init__(self, pool, slots):
        if pool.dim() != 4 or pool.shape[2] != pool.shape[3] or pool.dtype != torch.float32 or not pool.is_contiguous():
            raise ValueError("pool must be contiguous f32 [num_slots][num_kv_heads][head_dim][head_dim]")
        self.pool = pool
        if isinstance(slots, tuple):
            self.slots_host, self.slots = slots
        else:
            self.slots_host = torch.as_tensor(slots, dtype=torch.int32).cpu().contiguous()
            self.slots = self.slots_host.to(pool.device)

    @classmethod
    def allocate(cls, num_slots, num_kv_heads, head_dim, slots, device="cuda"):
        """New states, zero: sessions at their beginning."""
        return cls(torch.zeros((num_slots, num_kv_heads, head_dim, head_dim), dtype=torch.float32, device=device), slots)

    def desc(self):
        slots, heads, dim = self.pool.shape[:3]
        return LinearStateDesc(self.pool.data_ptr(), self.slots.data_ptr(), self.slots_host.data_ptr(), slots, heads, dim)


def linear_workspace_bytes(num_seqs, total_tokens, num_q_heads, num_kv_heads, head_dim):
    """Workspace bytes of a packed call and of its gradients."""
    return library().ws_linear_workspace_bytes(num_seqs, total_tokens, num_q_heads, num_kv_heads, head_dim)


def _check_decay(log_decay, hkv):
    _shape("log_decay", log_decay, (hkv,))
    if log_decay.dtype != torch.float32 or not log_decay.is_contiguous():
        raise ValueError("log_decay must be contiguous f32")


def _check_state(state, count):
    if not isinstance(state, LinearState):
        raise ValueError("state must be a LinearState")
    if tuple(state.slots_host.shape) != (count,) or tuple(state.slots.shape) != (count,):
        raise ValueError(f"state must have {count} slots")
    _check_pair("slots", state.slots_host, state.slots)
    pool = state.pool
    if not _here(pool) or pool.dim() != 4 or pool.shape[2] != pool.shape[3] or pool.dtype != torch.float32 or not pool.is_contiguous():
        raise ValueError("state pool must be contiguous f32 [num_slots][num_kv_heads][head_dim][head_dim] on the current device")


def _check_states(name, t, shape):
    _shape(name, t, shape)
    if t is not None and (t.dtype != torch.float32 or not t.is_contiguous()):
        raise ValueError(f"{name} must be contiguous f32")


def linear_attn_prefill(q, k, v, log_decay, seq_offsets, scale=None, state=None, reset=False, commit=True, out=None,
                        out_dtype=torch.bfloat16, workspace=None):
    """Packed sequences: q [T][Hq][d]; k, v [T][Hkv][d]; log_decay f32 [Hkv];
    sequence s is the tokens [seq_offsets[s], seq_offsets[s + 1]) (array-like, or
    a (host, device) pair).  scale: 1 / sqrt(d) by default.
    state (a LinearState of as many slots as sequences): sequences begin with
    their states (reset: with zero) and leave theirs (commit=False: do not).
    Returns out [T][Hq][d]; rows behind the last sequence are not written."""
    got = _native().linear_prefill(q, k, v, log_decay, seq_offsets, scale, state, reset, commit, out, out_dtype, workspace)
    if got is not None:
        if got[0]:
            _check(got[0])
        return got[1]
    T, Hq, D = q.shape
    hkv = k.shape[1]
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    off_h, off_d, n = _seq_offsets(seq_offsets, q.device)
    if out is None:
        out = torch.empty((T, Hq, D), dtype=out_dtype, device=q.device)
    for name, t, heads in (("q", q, Hq), ("k", k, hkv), ("v", v, hkv), ("out", out, Hq)):
        _shape(name, t, (T, heads, D))
    _check_decay(log_decay, hkv)
    if state is not None:
        _check_state(state, n)
    workspace, size = _workspace(workspace, linear_workspace_bytes(n, T, Hq, hkv, D), q.device)
    desc = ctypes.byref(state.desc()) if state is not None else None
    flags = (WS_STATE_RESET if reset else 0) | (0 if commit else WS_STATE_KEEP)
    _check(library().ws_linear_attn_prefill(_t3(q), _t3(k), _t3(v), _ptr(log_decay), off_h.data_ptr(), off_d.data_ptr(), n, T,
                                            Hq, hkv, D, float(scale), desc, flags, _t3(out), _ptr(workspace), size, _stream()))
    return out


def linear_attn_step(q, k, v, log_decay, state, scale=None, commit=True, new_lens=None, out=None, out_dtype=torch.bfloat16):
    """A few new tokens of each session against its state, the recurrent form:
    q [B][Ln][Hq][d]; k, v [B][Ln][Hkv][d].  The states are advanced in place
    (commit=False: left, so that a noisy block can be tried).  new_lens
    (optional, [B], 0..Ln): tokens of each; rows past them are not written.
    From some tens of tokens on ``linear_attn_prefill`` is faster."""
    got = _native().linear_step(q, k, v, log_decay, state, scale, commit, new_lens, out, out_dtype)
    if got is not None:
        if got[0]:
            _check(got[0])
        return got[1]
    B, Ln, Hq, D = q.shape
    hkv = k.shape[2]
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if out is None:
        out = torch.empty((B, Ln, Hq, D), dtype=out_dtype, device=q.device)
    for name, t, heads in (("q", q, Hq), ("k", k, hkv), ("v", v, hkv), ("out", out, Hq)):
        _shape(name, t, (B, Ln, heads, D))
    _check_decay(log_decay, hkv)
    _check_state(state, B)
    if tuple(state.pool.shape[1:]) != (hkv, D, D):
        raise ValueError("state heads or head_dim differ from the keys'")
    nh, nd = (None, None) if new_lens is None else _int32_pair(new_lens, (B,), q.device)
    desc = state.desc()
    _check(library().ws_linear_attn_step(_t4(q), _t4(k), _t4(v), _ptr(log_decay), ctypes.byref(desc), _ptr(nh), _ptr(nd), B, Ln,
                                         Hq, float(scale), 0 if commit else WS_STATE_KEEP, _t4(out), _stream()))
    return out


def linear_attn_prefill_bwd(q, k, v, dout, log_decay, seq_offsets, scale=None, state=None, dstate=None, want_dstate0=False,
                            dq=None, dk=None, dv=None, dstate0=None, workspace=None):
    """Gradients of ``linear_attn_prefill`` for an upstream dout [T][Hq][d] (and
    dstate, f32 [S][Hkv][d][d], of the final states): bf16 (dq [T][Hq][d], dk, dv
    [T][Hkv][d]), and with want_dstate0 the f32 gradient of the first states.
    state: the states the sequences began with (read only; None: zero)."""
    want_dstate0 = want_dstate0 or dstate0 is not None
    got = _native().linear_bwd(q, k, v, dout, log_decay, seq_offsets, scale, state, dstate, want_dstate0, dq, dk, dv, dstate0,
                               workspace)
    if got is not None:
        if got[0]:
            _check(got[0])
        return got[1:] if want_dstate0 else got[1:4]
    T, Hq, D = q.shape
    hkv = k.shape[1]
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    off_h, off_d, n = _seq_offsets(seq_offsets, q.device)
    dq = torch.empty((T, Hq, D), dtype=torch.bfloat16, device=q.device) if dq is None else dq
    dk = torch.empty((T, hkv, D), dtype=torch.bfloat16, device=q.device) if dk is None else dk
    dv = torch.empty((T, hkv, D), dtype=torch.bfloat16, device=q.device) if dv is None else dv
    for name, t, heads in (("q", q, Hq), ("k", k, hkv), ("v", v, hkv), ("dout", dout, Hq), ("dq", dq, Hq), ("dk", dk, hkv),
                           ("dv", dv, hkv)):
        _shape(name, t, (T, heads, D))
    _check_decay(log_decay, hkv)
    if state is not None:
        _check_state(state, n)
    if want_dstate0 and dstate0 is None:
        dstate0 = torch.empty((n, hkv, D, D), dtype=torch.float32, device=q.device)
    _check_states("dstate", dstate, (n, hkv, D, D))
    _check_states("dstate0", dstate0, (n, hkv, D, D))
    workspace, size = _workspace(workspace, linear_workspace_bytes(n, T, Hq, hkv, D), q.device)
    desc = ctypes.byref(state.desc()) if state is not None else None
    _check(library().ws_linear_attn_prefill_bwd(_t3(q), _t3(k), _t3(v), _t3(dout), _ptr(log_decay), off_h.data_ptr(),
                                                off_d.data_ptr(), n, T, Hq, hkv, D, float(scale), desc, _ptr(dstate),
                                                _ptr(dstate0), _t3(dq), _t3(dk), _t3(dv), _ptr(workspace), size, _stream()))
    return (dq, dk, dv, dstate0) if want_dstate0 else (dq, dk, dv)
