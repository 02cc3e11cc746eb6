"""Operators of sequence models (include/nugpr.h has their definitions): same names as the C entry points, argument checks and
marshalling only.  Arrays are CUDA tensors, float32 or bfloat16, of any strides with the last dimension contiguous; offsets,
slots and the like stay on the device, and no call waits for the GPU.  Outputs and scratch memory are torch tensors on
the current stream of the tensors' device."""
from __future__ import annotations

import ctypes as C

from .binding import (Adapter, DecayAttention, Heads, NUGPR_BFLOAT16, NUGPR_ERR_INVALID, NUGPR_FLOAT32, NugprError,
                      _check, load_library)


def _refuse(what):
    raise NugprError(NUGPR_ERR_INVALID, what)


def _types():
    import torch
    return torch, {torch.float32: NUGPR_FLOAT32, torch.bfloat16: NUGPR_BFLOAT16}


def _tensor(t, name, like, shape, dtype):
    """`t` as it is, or a refusal: on `like`'s device, of this shape (None: any) and type."""
    if t.device != like.device or not t.is_cuda:
        _refuse(f"{name} must be on the GPU that q or x is on")
    if t.dtype != dtype:
        _refuse(f"{name} must be {dtype}, not {t.dtype}")
    if t.dim() != len(shape) or any(w is not None and w != s for w, s in zip(shape, t.shape)):
        _refuse(f"{name} must have the shape {tuple('any' if w is None else w for w in shape)}, not {tuple(t.shape)}")
    return t


def _dense(t, name, like, shape, dtype):
    if not _tensor(t, name, like, shape, dtype).is_contiguous():
        _refuse(f"{name} must be contiguous")
    return t


def _inner(t, name):
    if t.stride(-1) != 1 and t.shape[-1] > 1 and t.numel():
        _refuse(f"the last dimension of {name} must be contiguous")


def _heads(t, name):
    _inner(t, name)
    return Heads(t.data_ptr(), t.stride(0), t.stride(1))


def _stream(torch, device):
    return torch.cuda.current_stream(device).cuda_stream


def _attention(q, k, v, log_decay, scale):
    """The problem's structure with everything but sequences and workspace."""
    torch, types = _types()
    if q.dtype not in types:
        _refuse(f"q must be float32 or bfloat16, not {q.dtype}")
    if q.dim() != 3:
        _refuse("q must be rows x heads x dim_k")
    n = q.shape[0]
    _tensor(q, "q", q, (n, None, None), q.dtype)
    _tensor(k, "k", q, (n, None, q.shape[2]), q.dtype)
    _tensor(v, "v", q, (n, k.shape[1], None), q.dtype)
    _dense(log_decay, "log_decay", q, (k.shape[1],), torch.float32)
    p = DecayAttention()
    p.dtype, p.heads, p.kv_heads, p.dim_k, p.dim_v = types[q.dtype], q.shape[1], k.shape[1], q.shape[2], v.shape[2]
    p.n_rows, p.log_decay = n, log_decay.data_ptr()
    p.scale = float(scale)
    return torch, p


def _sequences(torch, p, q, seq_offsets, backward):
    """Puts offsets and scratch memory into the problem; returns what has to stay alive during the call."""
    _dense(seq_offsets, "seq_offsets", q, (None,), torch.int64)
    if seq_offsets.shape[0] < 1:
        _refuse("seq_offsets must have n_seqs + 1 entries")
    p.n_seqs, p.seq_offsets = seq_offsets.shape[0] - 1, seq_offsets.data_ptr()
    need = load_library().nugpr_decay_attention_workspace_bytes(C.byref(p), backward)
    if need == 0:
        raise NugprError(NUGPR_ERR_INVALID, load_library().nugpr_last_error_string().decode())
    ws = torch.empty(need, dtype=torch.uint8, device=q.device)       # (torch aligns allocations to 512 bytes)
    p.workspace, p.workspace_bytes = ws.data_ptr(), need
    return ws


def _state(t, name, q, p, torch):
    if t is None:
        return None
    return _dense(t, name, q, (p.n_seqs, p.kv_heads, p.dim_k, p.dim_v), torch.float32).data_ptr()


def nugpr_decay_attention_forward(q, k, v, log_decay, seq_offsets, scale=1.0, initial_state=None):
    """Linear attention with a decay for each head over packed sequences.

    q (rows, heads, dim_k), k (rows, kv_heads, dim_k), v (rows, kv_heads, dim_v): float32 or bfloat16; log_decay (kv_heads,)
    float32, <= 0; seq_offsets (n_seqs + 1,) int64; initial_state (n_seqs, kv_heads, dim_k, dim_v) float32 or None.
    Returns o (rows, heads, dim_v) and the sequences' end states, float32."""
    torch, p = _attention(q, k, v, log_decay, scale)
    ws = _sequences(torch, p, q, seq_offsets, 0)  # noqa: F841
    s0 = _state(initial_state, "initial_state", q, p, torch)
    o = torch.empty((q.shape[0], p.heads, p.dim_v), dtype=q.dtype, device=q.device)
    s1 = torch.empty((p.n_seqs, p.kv_heads, p.dim_k, p.dim_v), dtype=torch.float32, device=q.device)
    with torch.cuda.device(q.device):
        _check(load_library().nugpr_decay_attention_forward(
            C.byref(p), C.byref(_heads(q, "q")), C.byref(_heads(k, "k")), C.byref(_heads(v, "v")), s0,
            C.byref(_heads(o, "o")), s1.data_ptr(), _stream(torch, q.device)))
    return o, s1


def nugpr_decay_attention_backward(q, k, v, log_decay, seq_offsets, d_o, scale=1.0, initial_state=None,
                                   d_final_state=None):
    """Gradients of nugpr_decay_attention_forward's q, k, v (in their type) and initial state (float32), from d_o and, unless
    None, d_final_state."""
    torch, p = _attention(q, k, v, log_decay, scale)
    ws = _sequences(torch, p, q, seq_offsets, 1)  # noqa: F841
    s0 = _state(initial_state, "initial_state", q, p, torch)
    s1 = _state(d_final_state, "d_final_state", q, p, torch)
    _tensor(d_o, "d_o", q, (q.shape[0], p.heads, p.dim_v), q.dtype)
    dq, dk, dv = (torch.empty(t.shape, dtype=q.dtype, device=q.device) for t in (q, k, v))
    ds = torch.empty((p.n_seqs, p.kv_heads, p.dim_k, p.dim_v), dtype=torch.float32, device=q.device)
    with torch.cuda.device(q.device):
        _check(load_library().nugpr_decay_attention_backward(
            C.byref(p), C.byref(_heads(q, "q")), C.byref(_heads(k, "k")), C.byref(_heads(v, "v")), s0,
            C.byref(_heads(d_o, "d_o")), s1, C.byref(_heads(dq, "dq")), C.byref(_heads(dk, "dk")),
            C.byref(_heads(dv, "dv")), ds.data_ptr(), _stream(torch, q.device)))
    return dq, dk, dv, ds


def nugpr_decay_attention_step(q, k, v, log_decay, state, slots=None, scale=1.0):
    """One token for each request: q (requests, heads, dim_k), k, v alike; state (n_states, kv_heads, dim_k, dim_v) float32 is
    advanced in place, request b's at slots[b] (int32; None: b).  Returns o (requests, heads, dim_v)."""
    torch, p = _attention(q, k, v, log_decay, scale)
    p.n_seqs = state.shape[0] if state.dim() == 4 else 0
    st = _state(state, "state", q, p, torch)
    if slots is not None:
        _dense(slots, "slots", q, (q.shape[0],), torch.int32)
    o = torch.empty((q.shape[0], p.heads, p.dim_v), dtype=q.dtype, device=q.device)
    with torch.cuda.device(q.device):
        _check(load_library().nugpr_decay_attention_step(
            C.byref(p), C.byref(_heads(q, "q")), C.byref(_heads(k, "k")), C.byref(_heads(v, "v")), st,
            None if slots is None else slots.data_ptr(), C.byref(_heads(o, "o")), _stream(torch, q.device)))
    return o


def _adapter(x, W, A, B, offsets, adapter_of, scale, backward):
    """The problem's structure and what has to stay alive during the call."""
    torch, types = _types()
    if x.dtype not in types:
        _refuse(f"x must be float32 or bfloat16, not {x.dtype}")
    if W.dim() != 2 or A.dim() != 3:
        _refuse("W must be dim_out x dim_in and A adapters x rank x dim_in")
    _tensor(x, "x", x, (None, W.shape[1]), x.dtype)
    _inner(x, "x")
    _dense(W, "W", x, (None, None), x.dtype)
    _dense(A, "A", x, (None, None, W.shape[1]), x.dtype)
    _dense(B, "B", x, (A.shape[0], A.shape[1], W.shape[0]), x.dtype)
    _dense(offsets, "seq_offsets", x, (None,), torch.int64)
    if offsets.shape[0] < 1:
        _refuse("seq_offsets must have n_seqs + 1 entries")
    p = Adapter()
    p.dtype, p.dim_in, p.dim_out, p.rank, p.n_adapters = types[x.dtype], W.shape[1], W.shape[0], A.shape[1], A.shape[0]
    p.n_rows, p.n_seqs, p.seq_offsets = x.shape[0], offsets.shape[0] - 1, offsets.data_ptr()
    if adapter_of is not None:
        p.adapter_of = _dense(adapter_of, "adapter_of", x, (p.n_seqs,), torch.int32).data_ptr()
    p.W, p.A, p.B, p.scale = W.data_ptr(), A.data_ptr(), B.data_ptr(), float(scale)
    need = load_library().nugpr_adapter_workspace_bytes(C.byref(p), backward)
    if need == 0:
        raise NugprError(NUGPR_ERR_INVALID, load_library().nugpr_last_error_string().decode())
    ws = torch.empty(need, dtype=torch.uint8, device=x.device)
    p.workspace, p.workspace_bytes = ws.data_ptr(), need
    return torch, p, ws


def nugpr_adapter_forward(x, W, A, B, seq_offsets, adapter_of=None, scale=1.0):
    """y = x W^T + scale (x A_a^T) B_a, a = adapter_of[s] (None: s) for the rows seq_offsets[s] .. seq_offsets[s + 1] - 1.

    x (rows, dim_in), W (dim_out, dim_in), A (adapters, rank, dim_in), B (adapters, rank, dim_out): float32 or bfloat16, W, A
    and B contiguous; seq_offsets (n_seqs + 1,) int64; adapter_of (n_seqs,) int32.  Returns y (rows, dim_out)."""
    torch, p, ws = _adapter(x, W, A, B, seq_offsets, adapter_of, scale, 0)
    y = torch.empty((x.shape[0], p.dim_out), dtype=x.dtype, device=x.device)
    with torch.cuda.device(x.device):
        _check(load_library().nugpr_adapter_forward(C.byref(p), x.data_ptr(), x.stride(0), y.data_ptr(),
                                                    _stream(torch, x.device)))
    return y


def nugpr_adapter_backward(x, W, A, B, seq_offsets, d_y, adapter_of=None, scale=1.0):
    """Gradients of nugpr_adapter_forward's x, A and B, in their type, from d_y; W is fixed."""
    torch, p, ws = _adapter(x, W, A, B, seq_offsets, adapter_of, scale, 1)
    _tensor(d_y, "d_y", x, (x.shape[0], p.dim_out), x.dtype)
    _inner(d_y, "d_y")
    dx = torch.empty((x.shape[0], p.dim_in), dtype=x.dtype, device=x.device)
    dA, dB = torch.empty_like(A), torch.empty_like(B)
    with torch.cuda.device(x.device):
        _check(load_library().nugpr_adapter_backward(C.byref(p), x.data_ptr(), x.stride(0), d_y.data_ptr(), d_y.stride(0),
                                                     dx.data_ptr(), dA.data_ptr(), dB.data_ptr(), _stream(torch, x.device)))
    return dx, dA, dB
