"""CPU-side checks of the sequence operators' C entry points: sizes of workspaces, and refusals before any GPU work."""
import ctypes as C
import os

import pytest

from paper_2510_12128_amd import binding as B


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.lib_path()):
        from paper_2510_12128_amd import build
        build.build()
    return B.load_library()


def attention(**kw):
    p = B.DecayAttention(dtype=B.NUGPR_FLOAT32, heads=4, kv_heads=2, dim_k=64, dim_v=32, n_rows=1000, n_seqs=3,
                         seq_offsets=4096, log_decay=4096, scale=1.0, workspace=4096, workspace_bytes=1 << 40)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def adapter(**kw):
    p = B.Adapter(dtype=B.NUGPR_BFLOAT16, dim_in=64, dim_out=48, rank=8, n_adapters=2, n_rows=100, n_seqs=3, seq_offsets=4096,
                  adapter_of=None, W=4096, A=4096, B=4096, scale=1.0, workspace=4096, workspace_bytes=1 << 40)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


BAD_ATTENTION = [dict(dtype=2), dict(heads=3), dict(heads=0), dict(kv_heads=0), dict(kv_heads=-1), dict(dim_k=0), dict(dim_k=129),
                 dict(dim_v=129), dict(n_rows=-1), dict(n_seqs=-1), dict(heads=8192, kv_heads=8192)]
BAD_ADAPTER = [dict(dtype=-1), dict(dim_in=0), dict(dim_out=65537), dict(rank=0), dict(rank=129), dict(n_adapters=-1),
               dict(n_adapters=1 << 16), dict(n_rows=-1), dict(n_seqs=-1)]


def test_workspace_sizes(lib):
    small = lib.nugpr_decay_attention_workspace_bytes(C.byref(attention()), 0)
    assert small > 0 and small % 256 == 0
    assert lib.nugpr_decay_attention_workspace_bytes(C.byref(attention()), 1) > small
    # a state for every piece of a sequence, never more than a few hundred beside one for each sequence
    one = 4 * 2 * 64 * 32
    assert lib.nugpr_decay_attention_workspace_bytes(C.byref(attention(n_rows=1 << 30)), 0) < 1100 * one
    a = lib.nugpr_adapter_workspace_bytes(C.byref(adapter()), 0)
    assert a >= 100 * 32 * 4 and a % 256 == 0
    assert lib.nugpr_adapter_workspace_bytes(C.byref(adapter()), 1) >= 2 * 100 * 32 * 4


@pytest.mark.parametrize("kw", BAD_ATTENTION, ids=str)
def test_bad_attention_problems(lib, kw):
    p = attention(**kw)
    h = B.Heads(4096, 64, 64)
    assert lib.nugpr_decay_attention_workspace_bytes(C.byref(p), 0) == 0
    assert len(lib.nugpr_last_error_string()) > 0
    assert lib.nugpr_decay_attention_forward(C.byref(p), h, h, h, None, h, None, None) == B.NUGPR_ERR_INVALID
    assert lib.nugpr_decay_attention_backward(C.byref(p), h, h, h, None, h, None, h, h, h, None, None) == B.NUGPR_ERR_INVALID
    assert lib.nugpr_decay_attention_step(C.byref(p), h, h, h, 4096, None, h, None) == B.NUGPR_ERR_INVALID


def test_gradients_of_states_that_overlap_are_refused(lib):
    h, p = B.Heads(4096, 64, 64), attention(workspace_bytes=1 << 40)
    size = 3 * 2 * 64 * 32 * 4

    def backward(d_final, d_initial):
        return lib.nugpr_decay_attention_backward(C.byref(p), h, h, h, None, h, d_final, h, h, h, d_initial, None)

    for apart in (0, 4, size - 4):
        assert backward(1 << 20, (1 << 20) + apart) == B.NUGPR_ERR_INVALID
        assert backward((1 << 20) + apart, 1 << 20) == B.NUGPR_ERR_INVALID
        assert b"overlaps" in lib.nugpr_last_error_string()


def test_bad_attention_calls(lib):
    h, null, odd, back = B.Heads(4096, 64, 64), B.Heads(None, 64, 64), B.Heads(4098, 64, 64), B.Heads(4096, -64, 64)

    def forward(p, *heads):
        return lib.nugpr_decay_attention_forward(C.byref(p), heads[0], heads[1], heads[2], None, heads[3], None, None)

    for x in (null, odd, back):
        for at in range(4):
            heads = [h] * 4
            heads[at] = x
            assert forward(attention(), *heads) == B.NUGPR_ERR_INVALID
    assert forward(attention(), None, h, h, h) == B.NUGPR_ERR_INVALID
    assert forward(attention(scale=float("nan")), h, h, h, h) == B.NUGPR_ERR_INVALID
    assert forward(attention(seq_offsets=None), h, h, h, h) == B.NUGPR_ERR_INVALID
    assert forward(attention(log_decay=None), h, h, h, h) == B.NUGPR_ERR_INVALID
    assert forward(attention(n_seqs=0), h, h, h, h) == B.NUGPR_ERR_INVALID
    assert forward(attention(workspace=None), h, h, h, h) == B.NUGPR_ERR_WORKSPACE
    assert forward(attention(workspace=4097), h, h, h, h) == B.NUGPR_ERR_WORKSPACE
    assert forward(attention(workspace_bytes=10), h, h, h, h) == B.NUGPR_ERR_WORKSPACE
    assert lib.nugpr_decay_attention_forward(None, h, h, h, None, h, None, None) == B.NUGPR_ERR_INVALID
    step = lib.nugpr_decay_attention_step
    assert step(C.byref(attention()), h, h, h, 4096, None, h, None) == B.NUGPR_ERR_INVALID        # 1000 requests, 3 states
    assert step(C.byref(attention(n_rows=2)), h, h, h, None, None, h, None) == B.NUGPR_ERR_INVALID
    assert step(C.byref(attention(n_rows=2)), h, h, h, 4097, None, h, None) == B.NUGPR_ERR_INVALID
    assert step(C.byref(attention(n_rows=0)), h, h, h, None, None, h, None) == B.NUGPR_OK
    assert forward(attention(n_rows=0, n_seqs=0), h, h, h, h) == B.NUGPR_OK


@pytest.mark.parametrize("kw", BAD_ADAPTER, ids=str)
def test_bad_adapter_problems(lib, kw):
    p = adapter(**kw)
    assert lib.nugpr_adapter_workspace_bytes(C.byref(p), 1) == 0
    assert lib.nugpr_adapter_forward(C.byref(p), 4096, 64, 4096, None) == B.NUGPR_ERR_INVALID
    assert lib.nugpr_adapter_backward(C.byref(p), 4096, 64, 4096, 48, 4096, 4096, 4096, None) == B.NUGPR_ERR_INVALID


def test_bad_adapter_calls(lib):
    f, b = lib.nugpr_adapter_forward, lib.nugpr_adapter_backward
    for kw in (dict(W=None), dict(A=None), dict(B=None), dict(W=4097), dict(seq_offsets=None), dict(scale=float("inf"))):
        assert f(C.byref(adapter(**kw)), 4096, 64, 4096, None) == B.NUGPR_ERR_INVALID
    for kw in (dict(workspace=None), dict(workspace=4097), dict(workspace_bytes=10)):
        assert f(C.byref(adapter(**kw)), 4096, 64, 4096, None) == B.NUGPR_ERR_WORKSPACE
    p = adapter()
    assert f(None, 4096, 64, 4096, None) == B.NUGPR_ERR_INVALID
    for args in ((None, 64, 4096), (4097, 64, 4096), (4096, -1, 4096), (4096, 64, None), (4096, 64, 4097)):
        assert f(C.byref(p), *args, None) == B.NUGPR_ERR_INVALID
    for at in (0, 2, 5, 6):
        args = [4096, 64, 4096, 48, 4096, 4096, 4096]
        args[at] = None
        assert b(C.byref(p), *args, None) == B.NUGPR_ERR_INVALID
    assert f(C.byref(adapter(n_rows=0)), None, 64, None, None) == B.NUGPR_OK
