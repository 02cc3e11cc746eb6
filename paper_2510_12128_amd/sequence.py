"""Operators of sequence models (include/nugpr.h has their definitions): same names as the C entry points, argument checks and
marshalling only.  Arrays are CUDA tensors, float32 or bfloat16, of any strides with the last dimension contiguous; offsets,
slots and the like stay on the device, and no call waits for the GPU.  Outputs and scratch memory are torch tensors on
the current stream of the tensors' device.  Autograd does not record the calls (their gradients are the _backward calls, for a
torch.autograd.Function or by hand): inputs that require gradients are refused where it would."""
from __future__ import annotations

import ctypes as C
from array import array
from operator import attrgetter

import torch

from .binding import (Adapter, DecayAttention, Heads, NUGPR_BFLOAT16, NUGPR_ERR_INVALID, NUGPR_FLOAT32,
                      NugprError, Rows, SelectiveScan, ShortConv, _check, load_library)

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


# (The checks of the operators below ask for a tensor's GPU by its number: a call with single tokens is as long as its checks.)
def _array(t, name, device, dtype, shape):
    """A rows x width array of that device, type and shape, with its last dimension contiguous."""
    if not (t.dtype is dtype and t.get_device() == device.index and t.shape == shape):
        _like(t, name, device, dtype, shape)
    s = t.stride()
    if s[1] != 1 and shape[1] > 1 and t.numel():
        _refuse(f"the last dimension of {name} must be contiguous")
    return _byref(Rows(t.data_ptr(), s[0]))


def _given(t, name, device, dtype, shape):
    """Address of a contiguous array that may be left out."""
    if t is None:
        return None
    if t.dtype is dtype and t.get_device() == device.index and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    return _dense(t, name, device, dtype, shape)


def _asked(*tensors):
    """Whether autograd expects to follow a gradient through one of the tensors."""
    if _recording():
        for t in tensors:
            if t is not None and t.requires_grad:
                return True
    return False


def _conv(x, weight, bias, silu, n_seqs, offsets):
    """The problem's structure, without workspace; device, type and the shape of the sequences' windows."""
    device, dtype = _first(x, "x", 2)
    if weight.dim() != 2:
        _refuse("weight must be dim x width")
    n, dim = x.shape
    width = weight.shape[1]
    w = _given(weight, "weight", device, dtype, (dim, width))
    b = _given(bias, "bias", device, dtype, (dim,))
    return (ShortConv(_TYPES[dtype], dim, width, 1 if silu else 0, n, n_seqs, offsets, w, b, None, 0), device, dtype,
            (n_seqs, max(width - 1, 0), dim))


def nugpr_short_conv_forward(x, weight, seq_offsets, bias=None, silu=False, initial_state=None):
    """Causal convolution along packed sequences, each channel by itself, with bias and x sigmoid(x) behind it where given.

    x (rows, dim), weight (dim, width), bias (dim,) or None: float32 or bfloat16; the last column of weight is the row's own;
    seq_offsets (n_seqs + 1,) int64; initial_state (n_seqs, width - 1, dim), the rows before each sequence, oldest first, or
    None: zero.  Returns y (rows, dim) and the last rows of the sequences, for a call that goes on."""
    lib = load_library()
    if _asked(x, weight, bias, initial_state):
        _refuse_recorded(x=x, weight=weight, bias=bias, initial_state=initial_state)
    p, device, dtype, shape = _conv(x, weight, bias, silu, *_offsets(seq_offsets, x.device))
    s0 = _given(initial_state, "initial_state", device, dtype, shape)
    y = torch.empty(x.shape, dtype=dtype, device=device)
    s1 = torch.empty(shape, dtype=dtype, device=device)
    _call(lib.nugpr_short_conv_forward, device, _byref(p), _byref(Rows(x.data_ptr(), _rows(x, "x"))), s0,
          _byref(Rows(y.data_ptr(), x.shape[1])), s1.data_ptr())
    return y, s1


def nugpr_short_conv_backward(x, weight, seq_offsets, d_y, bias=None, silu=False, initial_state=None, d_final_state=None):
    """Gradients of nugpr_short_conv_forward's x, weight, bias (None without one) and initial state, in their type, from d_y
    and, unless None, d_final_state."""
    lib = load_library()
    if _asked(x, weight, bias, d_y, initial_state, d_final_state):
        _refuse_recorded(x=x, weight=weight, bias=bias, d_y=d_y, initial_state=initial_state, d_final_state=d_final_state)
    p, device, dtype, shape = _conv(x, weight, bias, silu, *_offsets(seq_offsets, x.device))
    s0 = _given(initial_state, "initial_state", device, dtype, shape)
    s1 = _given(d_final_state, "d_final_state", device, dtype, shape)
    need = lib.nugpr_short_conv_workspace_bytes(_byref(p))
    if need == 0:
        raise NugprError(NUGPR_ERR_INVALID, lib.nugpr_last_error_string().decode())
    ws = torch.empty(need, dtype=torch.uint8, device=device)
    p.workspace, p.workspace_bytes = ws.data_ptr(), need
    dx, dw = torch.empty(x.shape, dtype=dtype, device=device), torch.empty_like(weight)
    db = None if bias is None else torch.empty_like(bias)
    ds = torch.empty(shape, dtype=dtype, device=device)
    _call(lib.nugpr_short_conv_backward, device, _byref(p), _byref(Rows(x.data_ptr(), _rows(x, "x"))), s0,
          _array(d_y, "d_y", device, dtype, x.shape), s1, _byref(Rows(dx.data_ptr(), x.shape[1])), dw.data_ptr(),
          None if db is None else db.data_ptr(), ds.data_ptr())
    return dx, dw, db, ds


def nugpr_short_conv_step(x, weight, state, slots=None, bias=None, silu=False):
    """One token for each request: x (requests, dim); state (n_states, width - 1, dim), of x's type, moves on by a row in
    place, request b's at slots[b] (int32; None: b).  Returns y (requests, dim)."""
    lib = load_library()
    if _asked(x, weight, bias, state):
        _refuse_recorded(x=x, weight=weight, bias=bias, state=state)
    p, device, dtype, shape = _conv(x, weight, bias, silu, state.shape[0] if state.dim() else 0, None)
    st = _given(state, "state", device, dtype, shape)
    at = _given(slots, "slots", device, torch.int32, (x.shape[0],))
    y = torch.empty(x.shape, dtype=dtype, device=device)
    _call(lib.nugpr_short_conv_step, device, _byref(p), _byref(Rows(x.data_ptr(), _rows(x, "x"))), st, at,
          _byref(Rows(y.data_ptr(), x.shape[1])))
    _written(state)
    return y


def _scan(x, dt, A, B, C, D, z, dt_bias, softplus, n_seqs, offsets):
    """The problem's structure, without workspace; device, type, the shape of the sequences' states, and the arrays x, dt, B,
    C and z as the calls take them."""
    device, dtype = _first(x, "x", 2)
    if A.dim() != 2 or B.dim() != 3:
        _refuse("A must be dim x dim_state, B and C rows x groups x dim_state")
    n, dim = rows = x.shape
    groups, states = B.shape[1], A.shape[1]
    if not (B.dtype is C.dtype is dtype and B.get_device() == C.get_device() == device.index and B.shape == C.shape and
            B.shape[0] == n and B.shape[2] == states):
        _like(B, "B", device, dtype, (n, groups, states))
        _like(C, "C", device, dtype, (n, groups, states))
    a = _given(A, "A", device, torch.float32, (dim, states))
    d = _given(D, "D", device, torch.float32, (dim,))
    bias = _given(dt_bias, "dt_bias", device, torch.float32, (dim,))
    p = SelectiveScan(_TYPES[dtype], dim, groups, states, 1 if softplus else 0, n, n_seqs, offsets, a, d, bias, None, 0)
    arrays = (_byref(Rows(x.data_ptr(), _rows(x, "x"))), _array(dt, "dt", device, dtype, rows), _heads(B, "B"),
              _heads(C, "C"), None if z is None else _array(z, "z", device, dtype, rows))
    return p, device, dtype, (n_seqs, dim, states), arrays


def nugpr_selective_scan_forward(x, dt, A, B, C, seq_offsets, D=None, z=None, dt_bias=None, softplus=True,
                                 initial_state=None):
    """State space layer whose decay depends on the token, over packed sequences: with d = softplus(dt + dt_bias) (without
    `softplus`: dt + dt_bias), h_t = exp(d_t A) h_t-1 + d_t x_t B_t for each channel, y_t = (C_t . h_t + D x_t) silu(z_t).

    x, dt, z (rows, dim), B, C (rows, groups, dim_state): float32 or bfloat16, channels in `groups` equal groups; A (dim,
    dim_state), <= 0, D and dt_bias (dim,): float32; z, D and dt_bias may be None; seq_offsets (n_seqs + 1,) int64, n_seqs at
    least 1 where there are rows; initial_state (n_seqs, dim, dim_state) float32 or None.  Returns y (rows, dim) and the
    sequences' end states, float32."""
    lib = load_library()
    if _asked(x, dt, A, B, C, D, z, dt_bias, initial_state):
        _refuse_recorded(x=x, dt=dt, A=A, B=B, C=C, D=D, z=z, dt_bias=dt_bias, initial_state=initial_state)
    p, device, dtype, shape, arrays = _scan(x, dt, A, B, C, D, z, dt_bias, softplus, *_offsets(seq_offsets, x.device))
    ws = _scratch(lib, lib.nugpr_selective_scan_workspace_bytes, p, 0, device)  # noqa: F841
    s0 = _given(initial_state, "initial_state", device, torch.float32, shape)
    y = torch.empty(x.shape, dtype=dtype, device=device)
    s1 = torch.empty(shape, dtype=torch.float32, device=device)
    _call(lib.nugpr_selective_scan_forward, device, _byref(p), *arrays, s0, _byref(Rows(y.data_ptr(), x.shape[1])),
          s1.data_ptr())
    return y, s1


def nugpr_selective_scan_backward(x, dt, A, B, C, seq_offsets, d_y, D=None, z=None, dt_bias=None, softplus=True,
                                  initial_state=None, d_final_state=None):
    """Gradients of nugpr_selective_scan_forward's x, dt, A, B, C, D, z, dt_bias and initial state, in this order and in their
    types (None for D, z and dt_bias that are None), from d_y and, unless None, d_final_state."""
    lib = load_library()
    if _asked(x, dt, A, B, C, d_y, D, z, dt_bias, initial_state, d_final_state):
        _refuse_recorded(x=x, dt=dt, A=A, B=B, C=C, d_y=d_y, D=D, z=z, dt_bias=dt_bias, initial_state=initial_state,
                         d_final_state=d_final_state)
    p, device, dtype, shape, arrays = _scan(x, dt, A, B, C, D, z, dt_bias, softplus, *_offsets(seq_offsets, x.device))
    ws = _scratch(lib, lib.nugpr_selective_scan_workspace_bytes, p, 1, device)  # noqa: F841
    s0 = _given(initial_state, "initial_state", device, torch.float32, shape)
    s1 = _given(d_final_state, "d_final_state", device, torch.float32, shape)
    dx, ddt = (torch.empty(x.shape, dtype=dtype, device=device) for _ in range(2))
    dB, dC = (torch.empty(B.shape, dtype=dtype, device=device) for _ in range(2))
    dz = None if z is None else torch.empty(x.shape, dtype=dtype, device=device)
    dA = torch.empty_like(A)
    dD, dbias = (None if t is None else torch.empty_like(t) for t in (D, dt_bias))
    ds = torch.empty(shape, dtype=torch.float32, device=device)

    def out(t):
        return None if t is None else _byref(Rows(t.data_ptr(), x.shape[1]))

    _call(lib.nugpr_selective_scan_backward, device, _byref(p), *arrays, s0,
          _array(d_y, "d_y", device, dtype, x.shape), s1, out(dx), out(ddt),
          _heads(dB, "dB"), _heads(dC, "dC"), out(dz), dA.data_ptr(),
          None if dD is None else dD.data_ptr(), None if dbias is None else dbias.data_ptr(), ds.data_ptr())
    return dx, ddt, dA, dB, dC, dD, dz, dbias, ds


def nugpr_selective_scan_step(x, dt, A, B, C, state, slots=None, D=None, z=None, dt_bias=None, softplus=True):
    """One token for each request: x, dt, z (requests, dim), B, C (requests, groups, dim_state); state (n_states, dim,
    dim_state) float32 is advanced in place, request b's at slots[b] (int32; None: b).  Returns y (requests, dim)."""
    lib = load_library()
    if _asked(x, dt, A, B, C, D, z, dt_bias, state):
        _refuse_recorded(x=x, dt=dt, A=A, B=B, C=C, D=D, z=z, dt_bias=dt_bias, state=state)
    p, device, dtype, shape, arrays = _scan(x, dt, A, B, C, D, z, dt_bias, softplus,
                                            state.shape[0] if state.dim() else 0, None)
    st = _given(state, "state", device, torch.float32, shape)
    at = _given(slots, "slots", device, torch.int32, (x.shape[0],))
    y = torch.empty(x.shape, dtype=dtype, device=device)
    _call(lib.nugpr_selective_scan_step, device, _byref(p), *arrays, st, at, _byref(Rows(y.data_ptr(), x.shape[1])))
    _written(state)
    return y


_type_of, _shape_of, _asks = attrgetter("dtype"), attrgetter("shape"), attrgetter("requires_grad")
_address, _count, _where, _contiguous = (torch.Tensor.data_ptr, torch.Tensor.numel, torch.Tensor.get_device,
                                         torch.Tensor.is_contiguous)


def _run_of_memory(t):
    """Whether the values of a tensor fill one run of memory, in any order of its dimensions."""
    expected = 1
    for stride, size in sorted((st, si) for st, si in zip(t.stride(), t.shape) if si != 1):
        if stride != expected:
            return False
        expected *= size
    return True


def _same_order(g, o):
    """Whether two tensors of one shape that fill a run of memory have their values in the same order."""
    return (g.is_contiguous() and o.is_contiguous()) or g.numel() == 0 or all(
        a == b for a, b, size in zip(g.stride(), o.stride(), g.shape) if size != 1)


def _on_one_gpu(tensors, index, what):
    for i, t in enumerate(tensors):
        if t.get_device() != index or t.dtype not in _TYPES:
            _refuse(f"{what} {i} must be on the GPU of the first gradient, float32 or bfloat16")


def _gradients(grads, out):
    """The tensors as an array of the structure, their number and their device.  (Checks go over all tensors at once: a model has
    hundreds.)"""
    grads = list(grads)
    if not grads:
        _refuse("there is no gradient")
    if not grads[0].is_cuda:
        _refuse("gradients must be on a GPU")
    device, index = grads[0].device, grads[0].get_device()
    types = list(map(_type_of, grads))
    if set(map(_where, grads)) != {index} or not _TYPES.keys() >= set(types):
        _on_one_gpu(grads, index, "gradient")
    dense = all(map(_contiguous, grads))
    if not dense:
        for i, g in enumerate(grads):
            if g.numel() and not _run_of_memory(g):
                _refuse(f"gradient {i} must fill one run of memory")
    words = array("q", bytes(32 * len(grads)))                     # data, out, count, the two types  (of lists: faster than of a map)
    words[0::4] = array("q", list(map(_address, grads)))
    words[2::4] = array("q", list(map(_count, grads)))
    codes = [_TYPES[t] for t in types]
    to = grads
    if out is not None:
        to = list(out)
        if len(to) != len(grads):
            _refuse("out must have as many tensors as there are gradients")
        out_types = list(map(_type_of, to))
        if set(map(_where, to)) != {index} or not _TYPES.keys() >= set(out_types):
            _on_one_gpu(to, index, "out")
        if (list(map(_shape_of, to)) != list(map(_shape_of, grads)) or
                not (dense and all(map(_contiguous, to))) and not all(map(_same_order, grads, to))):
            _refuse("tensors of out must have the gradients' shapes and strides")
        words[1::4] = array("q", list(map(_address, to)))
        codes = [c | _TYPES[t] << 32 for c, t in zip(codes, out_types)]
    words[3::4] = array("q", codes)
    if _recording() and (any(map(_asks, grads)) or any(map(_asks, to))):
        _refuse("a gradient requires a gradient itself, which autograd does not get through this call")
    return words, to, device


def _norm_call(lib, call, words, device, *args):
    table, n = words.buffer_info()[0], len(words) // 4
    need = lib.nugpr_gradient_norm_workspace_bytes(table, n)
    if need == 0:
        raise NugprError(NUGPR_ERR_INVALID, lib.nugpr_last_error_string().decode())
    ws = torch.empty(need, dtype=torch.uint8, device=device)
    norm = torch.empty((), dtype=torch.float32, device=device)
    _call(call, device, table, n, *args, norm.data_ptr(), ws.data_ptr(), need)
    return norm


def nugpr_gradient_norm(grads):
    """The 2-norm of all values of the tensors in `grads` (float32 or bfloat16, on one GPU, any of them of either type), as a
    float32 tensor without dimensions."""
    lib = load_library()
    words, _, device = _gradients(grads, None)
    return _norm_call(lib, lib.nugpr_gradient_norm, words, device)


def nugpr_clip_gradients(grads, max_norm, out=None):
    """The same, and multiplies every value by min(1, max_norm / norm): in place, or into the tensors in `out` (of the
    gradients' shapes and strides, float32 or bfloat16).  No tensor that is written may share memory with another."""
    lib = load_library()
    words, to, device = _gradients(grads, out)
    norm = _norm_call(lib, lib.nugpr_clip_gradients, words, device, float(max_norm))
    _written(to)
    return norm
