"""Attention over packed sequences: sequences of different lengths one behind the
other in one token axis, without padding (include/ws_attn.h states it).

As the rest of the package this is marshalling only; the native module takes
the common case, the ctypes code here the others, with the checks and errors.

  block_causal_prefill_packed(q, k, v, seq_offsets, block_offsets=None, ...)
  block_causal_prefill_packed_bwd(q, k, v, o, dout, lse, seq_offsets, ...): its gradients
  prefill_packed_bwd_workspace_bytes(total_tokens, num_q_heads, num_kv_heads)
"""
import ctypes
import math

import torch

from . import (WS_DTYPE_BF16, WS_DTYPE_F32, Tensor4, _check, _check_lse, _check_pair, _check_workspace, _int32_pair, _native, _ptr,
               _shape, _stream, library)


def declare(lib):
    """Argument types of the packed entry points."""
    P, I32, F, N, T = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t, Tensor4
    lib.ws_block_causal_prefill_packed.restype = ctypes.c_int
    lib.ws_block_causal_prefill_packed.argtypes = [T, T, T, P, P, P, P, P, P, I32, I32, I32, I32, I32, I32, F, T, P, P]
    lib.ws_block_causal_prefill_packed_bwd.restype = ctypes.c_int
    lib.ws_block_causal_prefill_packed_bwd.argtypes = [T, T, T, T, T, P, P, P, P, P, P, P, I32, I32, I32, I32, I32, I32, F, T, T, T,
                                                       P, N, P]
    lib.ws_prefill_packed_bwd_workspace_bytes.restype = N
    lib.ws_prefill_packed_bwd_workspace_bytes.argtypes = [I32, I32, I32]


def _t3(t):
    """Descriptor of a packed [T][H][d] tensor."""
    if t.dim() != 3 or t.stride(2) != 1:
        raise ValueError("packed tensors must be 3-d [T][H][d] with a contiguous last dim")
    if t.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"unsupported dtype {t.dtype}")
    return Tensor4(t.data_ptr(), WS_DTYPE_BF16 if t.dtype == torch.bfloat16 else WS_DTYPE_F32, 0, t.stride(0), t.stride(1))


def _seq_offsets(seq_offsets, device, name="seq_offsets"):
    """(host, device) int32 offsets and the number of what lies between them."""
    if isinstance(seq_offsets, tuple):
        host, dev = seq_offsets
    else:
        host = torch.as_tensor(seq_offsets, dtype=torch.int32).cpu().contiguous()
        dev = host.to(device)
    if host.dim() != 1 or len(host) < 1 or dev.shape != host.shape:
        raise ValueError(f"{name} must be a vector of one more than they delimit")
    _check_pair(name, host, dev)
    return host, dev, len(host) - 1


def _workspace(workspace, need, device):
    _check_workspace(workspace)
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=device)
    return workspace, workspace.numel() * workspace.element_size()


def _blocks(block_offsets, text_starts, device):
    """((host, device) block offsets, (host, device) segment starts, their number);
    None: causal."""
    if block_offsets is None:
        if text_starts is not None:
            raise ValueError("text_starts need block_offsets")
        return (None, None), (None, None), 0
    host, dev, nb = _seq_offsets(block_offsets, device, "block_offsets")
    return (host, dev), (None, None) if text_starts is None else _int32_pair(text_starts, (nb,), device), nb


def prefill_packed_bwd_workspace_bytes(total_tokens, num_q_heads, num_kv_heads):
    """Workspace bytes of the gradients of a packed call."""
    return library().ws_prefill_packed_bwd_workspace_bytes(total_tokens, num_q_heads, num_kv_heads)


def block_causal_prefill_packed(q, k, v, seq_offsets, block_offsets=None, scale=None, out=None, out_dtype=torch.bfloat16,
                                want_lse=False, lse=None, text_starts=None):
    """Packed sequences: q [T][Hq][d]; k, v [T][Hkv][d]; sequence s is the tokens
    [seq_offsets[s], seq_offsets[s + 1]) (array-like, or a (host, device) pair).
    A token sees its own sequence, causally; with block_offsets [nb + 1] (in the
    packed axis; every sequence begins at one) by the block-causal rule of
    ``block_causal_prefill``, with text_starts [nb] blocks end in token-causal
    segments.  Returns out [T][Hq][d] (and lse [Hq][T] f32 when want_lse); rows
    behind the last sequence are not written."""
    got = _native().packed_prefill(q, k, v, seq_offsets, block_offsets, scale, out, out_dtype, want_lse, lse, text_starts)
    if got is not None:
        rc, out, lse = got
        if rc:
            _check(rc)
        return (out, lse) if want_lse else out
    T, Hq, D = q.shape
    hkv = k.shape[1]
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    off_h, off_d, n = _seq_offsets(seq_offsets, q.device)
    (bh, bd), (th, td), nb = _blocks(block_offsets, text_starts, q.device)
    if out is None:
        out = torch.empty((T, Hq, D), dtype=out_dtype, device=q.device)
    if want_lse and lse is None:
        lse = torch.empty((Hq, T), dtype=torch.float32, device=q.device)
    for name, t, heads in (("q", q, Hq), ("k", k, hkv), ("v", v, hkv), ("out", out, Hq)):
        _shape(name, t, (T, heads, D))
    _check_lse(lse, (Hq, T))
    _check(library().ws_block_causal_prefill_packed(
        _t3(q), _t3(k), _t3(v), off_h.data_ptr(), off_d.data_ptr(), _ptr(bh), _ptr(bd), _ptr(th), _ptr(td), n, T, nb, Hq, hkv, D,
        float(scale), _t3(out), _ptr(lse), _stream()))
    return (out, lse) if want_lse else out


def block_causal_prefill_packed_bwd(q, k, v, o, dout, lse, seq_offsets, block_offsets=None, scale=None, text_starts=None,
                                    dq=None, dk=None, dv=None, workspace=None, grad_dtype=torch.float32):
    """Gradients of ``block_causal_prefill_packed`` for an upstream dout [T][Hq][d]:
    (dq [T][Hq][d], dk, dv [T][Hkv][d]), f32 or bf16 (grad_dtype; the f32 sums
    rounded once).  o and lse are the forward's.  f32 gradients have the accuracy
    of bf16 operands."""
    if grad_dtype not in (torch.float32, torch.bfloat16):
        raise ValueError(f"unsupported grad_dtype {grad_dtype}")
    got = _native().packed_bwd(q, k, v, o, dout, lse, seq_offsets, block_offsets, scale, text_starts, dq, dk, dv, workspace,
                               grad_dtype)
    if got is not None:
        if got[0]:
            _check(got[0])
        return got[1:]
    T, Hq, D = q.shape
    hkv = k.shape[1]
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    off_h, off_d, n = _seq_offsets(seq_offsets, q.device)
    (bh, bd), (th, td), nb = _blocks(block_offsets, text_starts, q.device)
    dq = torch.empty((T, Hq, D), dtype=grad_dtype, device=q.device) if dq is None else dq
    dk = torch.empty((T, hkv, D), dtype=grad_dtype, device=q.device) if dk is None else dk
    dv = torch.empty((T, hkv, D), dtype=grad_dtype, device=q.device) if dv is None else dv
    for name, t, heads in (("q", q, Hq), ("k", k, hkv), ("v", v, hkv), ("o", o, Hq), ("dout", dout, Hq), ("dq", dq, Hq),
                           ("dk", dk, hkv), ("dv", dv, hkv)):
        _shape(name, t, (T, heads, D))
    _check_lse(lse, (Hq, T))
    workspace, size = _workspace(workspace, prefill_packed_bwd_workspace_bytes(T, Hq, hkv) if T else 0, q.device)
    _check(library().ws_block_causal_prefill_packed_bwd(
        _t3(q), _t3(k), _t3(v), _t3(o), _t3(dout), _ptr(lse), off_h.data_ptr(), off_d.data_ptr(), _ptr(bh), _ptr(bd), _ptr(th),
        _ptr(td), n, T, nb, Hq, hkv, D, float(scale), _t3(dq), _t3(dk), _t3(dv), _ptr(workspace), size, _stream()))
    return dq, dk, dv
