"""Operators of sequence models (include/nugpr.h has their definitions): same names as the C entry points, argument checks and
marshalling only.  Arrays are CUDA tensors, float32 or bfloat16, of any strides with the last dimension contiguous; offsets,
slots and the like stay on the device, and no call waits for the GPU.  Outputs and scratch memory are torch tensors on
the current stream of the tensors' device.  Autograd does not record the calls (their gradients are the _backward calls, for a
torch.autograd.Function or by hand): inputs that require gradients are refused where it would."""
from __future__ import annotations

import ctypes as C

import torch

from .binding import (Adapter, DecayAttention, Heads, NUGPR_BFLOAT16, NUGPR_ERR_INVALID, NUGPR_FLOAT32, NugprError,
                      _check, load_library)

_TYPES = {torch.float32: NUGPR_FLOAT32, torch.bfloat16: NUGPR_BFLOAT16}
_byref = C.byref


def _refuse(what):
    raise NugprError(NUGPR_ERR_INVALID, what)


def _like(t, name, device, dtype, shape):
    """Refuses `t` unless it is on that device, of that type and shape."""
    if t.dtype is dtype and t.device == device and t.shape == shape:
        return
    if t.device != device:
        _refuse(f"{name} is on {t.device}, not on {device}")
    if t.dtype is not dtype:
        _refuse(f"{name} must be {dtype}, not {t.dtype}")
    _refuse(f"{name} must have the shape {tuple(shape)}, not {tuple(t.shape)}")


def _dense(t, name, device, dtype, shape):
    """The same, and contiguous; its address."""
    _like(t, name, device, dtype, shape)
    if not t.is_contiguous():
        _refuse(f"{name} must be contiguous")
    return t.data_ptr()


def _refuse_recorded(**tensors):
    """Refuses the tensor whose gradient autograd expects to follow through the call."""
    for name, t in tensors.items():
        if t is not None and t.requires_grad:
            _refuse(f"{name} requires a gradient, which autograd does not get through this call: use torch.no_grad(), and "
                    "the _backward calls")


_recording, _written = torch.is_grad_enabled, torch.autograd.graph.increment_version


def _heads(t, name):
    s = t.stride()
    if s[2] != 1 and t.shape[2] > 1 and t.numel():
        _refuse(f"the last dimension of {name} must be contiguous")
    return _byref(Heads(t.data_ptr(), s[0], s[1]))


def _rows(t, name):
    s = t.stride()
    if s[1] != 1 and t.shape[1] > 1 and t.numel():
        _refuse(f"the last dimension of {name} must be contiguous")
    return s[0]


def _first(t, name, dims):
    """Type and device of the call, from its first array."""
    if not t.is_cuda:
        _refuse(f"{name} must be on a GPU")
    if t.dtype not in _TYPES:
        _refuse(f"{name} must be float32 or bfloat16, not {t.dtype}")
    if t.dim() != dims:
        _refuse(f"{name} must have {dims} dimensions")
    return t.device, t.dtype


# (address of a device's current stream; without it through a Stream object, 1.7 us slower)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _call(function, device, *args):
    """The call on the current stream of `device`, which is made current for it."""
    if device.index == torch.cuda.current_device():
        return _check(function(*args, _raw_stream(device.index)))
    with torch.cuda.device(device):
        return _check(function(*args, _raw_stream(device.index)))


def _scratch(lib, size, p, backward, device):
    """Scratch memory of the problem; it has to stay alive until the call is made (the allocator keeps it for the stream)."""
    need = size(_byref(p), backward)
    if need == 0:
        raise NugprError(NUGPR_ERR_INVALID, lib.nugpr_last_error_string().decode())
    ws = torch.empty(need, dtype=torch.uint8, device=device)       # (torch aligns allocations to 512 bytes)
    p.workspace, p.workspace_bytes = ws.data_ptr(), need
    return ws


def _attention(q, k, v, log_decay, scale, n_seqs, offsets):
    """The problem's structure, without workspace; device, type and the shape of a sequence's states."""
    device, dtype = _first(q, "q", 3)
    if k.dim() != 3 or v.dim() != 3:
        _refuse("k and v must be rows x kv_heads x width")
    n, heads, dk = q.shape
    kv, dv = k.shape[1], v.shape[2]
    _like(k, "k", device, dtype, (n, kv, dk))
    _like(v, "v", device, dtype, (n, kv, dv))
    decay = _dense(log_decay, "log_decay", device, torch.float32, (kv,))
    return (DecayAttention(_TYPES[dtype], heads, kv, dk, dv, n, n_seqs, offsets, decay, scale, None, 0), device, dtype,
            (n_seqs, kv, dk, dv))


def _offsets(t, device):
    """Number of sequences and address of their offsets."""
    if t.dim() != 1 or t.shape[0] < 1:
        _refuse("seq_offsets must have n_seqs + 1 entries")
    return t.shape[0] - 1, _dense(t, "seq_offsets", device, torch.int64, t.shape)


def nugpr_decay_attention_forward(q, k, v, log_decay, seq_offsets, scale=1.0, initial_state=None):
    """Linear attention with a decay for each head over packed sequences.

    q (rows, heads, dim_k), k (rows, kv_heads, dim_k), v (rows, kv_heads, dim_v): float32 or bfloat16; log_decay (kv_heads,)
    float32, <= 0; seq_offsets (n_seqs + 1,) int64, n_seqs at least 1 where there are rows; initial_state (n_seqs, kv_heads,
    dim_k, dim_v) float32 or None.  Returns o (rows, heads, dim_v) and the sequences' end states,
    float32."""
    lib = load_library()
    if _recording() and (q.requires_grad or k.requires_grad or v.requires_grad or log_decay.requires_grad or
                         (initial_state is not None and initial_state.requires_grad)):
        _refuse_recorded(q=q, k=k, v=v, log_decay=log_decay, initial_state=initial_state)
    p, device, dtype, shape = _attention(q, k, v, log_decay, scale, *_offsets(seq_offsets, q.device))
    ws = _scratch(lib, lib.nugpr_decay_attention_workspace_bytes, p, 0, device)  # noqa: F841
    s0 = None if initial_state is None else _dense(initial_state, "initial_state", device, torch.float32, shape)
    o = torch.empty((q.shape[0], q.shape[1], v.shape[2]), dtype=dtype, device=device)
    s1 = torch.empty(shape, dtype=torch.float32, device=device)
    _call(lib.nugpr_decay_attention_forward, device, _byref(p), _heads(q, "q"), _heads(k, "k"), _heads(v, "v"), s0,
          _heads(o, "o"), s1.data_ptr())
    return o, s1


def nugpr_decay_attention_backward(q, k, v, log_decay, seq_offsets, d_o, scale=1.0, initial_state=None,
                                   d_final_state=None):
    """Gradients of nugpr_decay_attention_forward's q, k, v (in their type) and initial state (float32), from d_o and, unless
    None, d_final_state."""
    lib = load_library()
    if _recording() and (q.requires_grad or k.requires_grad or v.requires_grad or log_decay.requires_grad or
                         d_o.requires_grad or (initial_state is not None and initial_state.requires_grad) or
                         (d_final_state is not None and d_final_state.requires_grad)):
        _refuse_recorded(q=q, k=k, v=v, log_decay=log_decay, d_o=d_o, initial_state=initial_state,
                         d_final_state=d_final_state)
    p, device, dtype, shape = _attention(q, k, v, log_decay, scale, *_offsets(seq_offsets, q.device))
    ws = _scratch(lib, lib.nugpr_decay_attention_workspace_bytes, p, 1, device)  # noqa: F841
    s0 = None if initial_state is None else _dense(initial_state, "initial_state", device, torch.float32, shape)
    s1 = None if d_final_state is None else _dense(d_final_state, "d_final_state", device, torch.float32, shape)
    _like(d_o, "d_o", device, dtype, (q.shape[0], q.shape[1], v.shape[2]))
    dq, dk, dv = (torch.empty(t.shape, dtype=dtype, device=device) for t in (q, k, v))
    ds = torch.empty(shape, dtype=torch.float32, device=device)
    _call(lib.nugpr_decay_attention_backward, device, _byref(p), _heads(q, "q"), _heads(k, "k"), _heads(v, "v"), s0,
          _heads(d_o, "d_o"), s1, _heads(dq, "dq"), _heads(dk, "dk"), _heads(dv, "dv"), ds.data_ptr())
    return dq, dk, dv, ds


def nugpr_decay_attention_step(q, k, v, log_decay, state, slots=None, scale=1.0):
    """One token for each request: q (requests, heads, dim_k), k, v alike; state (n_states, kv_heads, dim_k, dim_v) float32 is
    advanced in place, request b's at slots[b] (int32; None: b).  Returns o (requests, heads, dim_v)."""
    lib = load_library()
    if _recording() and (q.requires_grad or k.requires_grad or v.requires_grad or log_decay.requires_grad or state.requires_grad):
        _refuse_recorded(q=q, k=k, v=v, log_decay=log_decay, state=state)
    p, device, dtype, shape = _attention(q, k, v, log_decay, scale, state.shape[0] if state.dim() else 0, None)
    st = _dense(state, "state", device, torch.float32, shape)
    at = None if slots is None else _dense(slots, "slots", device, torch.int32, (q.shape[0],))
    o = torch.empty((q.shape[0], q.shape[1], v.shape[2]), dtype=dtype, device=device)
    _call(lib.nugpr_decay_attention_step, device, _byref(p), _heads(q, "q"), _heads(k, "k"), _heads(v, "v"), st, at,
          _heads(o, "o"))
    _written(state)                                                # (whoever saved it for a backward pass is told)
    return o


def _adapter(lib, x, W, A, B, seq_offsets, adapter_of, scale, backward):
    """The problem's structure, its scratch memory, device and type."""
    device, dtype = _first(x, "x", 2)
    if W.dim() != 2 or A.dim() != 3:
        _refuse("W must be dim_out x dim_in and A adapters x rank x dim_in")
    out, inp = W.shape
    n, rank = A.shape[0], A.shape[1]
    _like(x, "x", device, dtype, (x.shape[0], inp))
    w = _dense(W, "W", device, dtype, (out, inp))
    a = _dense(A, "A", device, dtype, (n, rank, inp))
    b = _dense(B, "B", device, dtype, (n, rank, out))
    n_seqs, offsets = _offsets(seq_offsets, device)
    which = None if adapter_of is None else _dense(adapter_of, "adapter_of", device, torch.int32, (n_seqs,))
    p = Adapter(_TYPES[dtype], inp, out, rank, n, x.shape[0], n_seqs, offsets, which, w, a, b, scale, None, 0)
    return p, _scratch(lib, lib.nugpr_adapter_workspace_bytes, p, backward, device), device, dtype


def nugpr_adapter_forward(x, W, A, B, seq_offsets, adapter_of=None, scale=1.0):
    """y = x W^T + scale (x A_a^T) B_a, a = adapter_of[s] (None: s) for the rows seq_offsets[s] .. seq_offsets[s + 1] - 1.

    x (rows, dim_in), W (dim_out, dim_in), A (adapters, rank, dim_in), B (adapters, rank, dim_out): float32 or bfloat16, W, A
    and B contiguous; seq_offsets (n_seqs + 1,) int64; adapter_of (n_seqs,) int32.  Returns y (rows, dim_out)."""
    lib = load_library()
    if _recording() and (x.requires_grad or W.requires_grad or A.requires_grad or B.requires_grad):
        _refuse_recorded(x=x, W=W, A=A, B=B)
    p, ws, device, dtype = _adapter(lib, x, W, A, B, seq_offsets, adapter_of, scale, 0)
    y = torch.empty((x.shape[0], W.shape[0]), dtype=dtype, device=device)
    _call(lib.nugpr_adapter_forward, device, _byref(p), x.data_ptr(), _rows(x, "x"), y.data_ptr())
    return y


def nugpr_adapter_backward(x, W, A, B, seq_offsets, d_y, adapter_of=None, scale=1.0):
    """Gradients of nugpr_adapter_forward's x, A and B, in their type, from d_y; W is fixed."""
    lib = load_library()
    if _recording() and (x.requires_grad or W.requires_grad or A.requires_grad or B.requires_grad or d_y.requires_grad):
        _refuse_recorded(x=x, W=W, A=A, B=B, d_y=d_y)
    p, ws, device, dtype = _adapter(lib, x, W, A, B, seq_offsets, adapter_of, scale, 1)
    _like(d_y, "d_y", device, dtype, (x.shape[0], W.shape[0]))
    dx = torch.empty(x.shape, dtype=dtype, device=device)
    dA, dB = torch.empty_like(A), torch.empty_like(B)
    _call(lib.nugpr_adapter_backward, device, _byref(p), x.data_ptr(), _rows(x, "x"), d_y.data_ptr(), _rows(d_y, "d_y"),
          dx.data_ptr(), dA.data_ptr(), dB.data_ptr())
    return dx, dA, dB
