"""CPU-side checks of the sequence operators' ranges: what one launch cannot hold is refused before any GPU work."""
import ctypes as C

import pytest

from paper_2510_12128_amd import binding as B
from test_sequence_host import adapter, attention, lib  # noqa: F401


@pytest.mark.parametrize("dims", [(64, 64), (128, 64)])
def test_more_workgroups_than_a_launch_counts_threads(lib, dims):  # noqa: F811
    """2^32 threads of one launch: 2^24 workgroups of 256 for widths up to 64, 2^23 of 512 beyond."""
    h = B.Heads(4096, 128, 128)
    kv = 4
    most = (1 << (24 if dims[0] <= 64 else 23)) // kv
    p = attention(heads=kv, kv_heads=kv, dim_k=dims[0], dim_v=dims[1], n_rows=10, n_seqs=most, workspace_bytes=1 << 60)
    assert lib.nugpr_decay_attention_forward(C.byref(p), h, h, h, None, h, None, None) == B.NUGPR_ERR_INVALID
    assert b"too many" in lib.nugpr_last_error_string()
    assert lib.nugpr_decay_attention_backward(C.byref(p), h, h, h, None, h, None, h, h, h, None, None) == B.NUGPR_ERR_INVALID
    assert b"too many" in lib.nugpr_last_error_string()


def test_more_single_tokens_than_a_launch_counts_threads(lib):  # noqa: F811
    h = B.Heads(4096, 128, 128)
    p = attention(heads=4, kv_heads=4, dim_k=128, dim_v=128, n_rows=1 << 20, n_seqs=1 << 20)
    assert lib.nugpr_decay_attention_step(C.byref(p), h, h, h, 4096, None, h, None) == B.NUGPR_ERR_INVALID
    assert b"too many" in lib.nugpr_last_error_string()


def test_scales_beyond_float32(lib):  # noqa: F811
    """The kernels multiply in float32, where such a scale is infinite and makes NaN of zeros."""
    h = B.Heads(4096, 64, 64)
    for scale in (1e39, -1e300):
        p = attention(scale=scale, n_rows=2)
        assert lib.nugpr_decay_attention_forward(C.byref(p), h, h, h, None, h, None, None) == B.NUGPR_ERR_INVALID
        assert lib.nugpr_decay_attention_backward(C.byref(p), h, h, h, None, h, None, h, h, h, None, None) == B.NUGPR_ERR_INVALID
        assert lib.nugpr_decay_attention_step(C.byref(p), h, h, h, 4096, None, h, None) == B.NUGPR_ERR_INVALID
        p = adapter(scale=scale)
        assert lib.nugpr_adapter_forward(C.byref(p), 4096, 64, 4096, None) == B.NUGPR_ERR_INVALID
        assert lib.nugpr_adapter_backward(C.byref(p), 4096, 64, 4096, 48, 4096, 4096, 4096, None) == B.NUGPR_ERR_INVALID
