"""CPU-side checks of the C entry points of the short convolution, the selective scan and the gradients' norm: sizes of
workspaces, and refusals before any GPU work."""
import ctypes as C

import pytest

from paper_2510_12128_amd import binding as B
from test_sequence_host import lib  # noqa: F401

INVALID, WORKSPACE = B.NUGPR_ERR_INVALID, B.NUGPR_ERR_WORKSPACE
OK, NULL, ODD, BACK = B.Rows(4096, 64), B.Rows(None, 64), B.Rows(4098, 64), B.Rows(4096, -64)
H = B.Heads(4096, 32, 16)


def conv(**kw):
    p = B.ShortConv(dtype=B.NUGPR_FLOAT32, dim=64, width=4, silu=1, n_rows=1000, n_seqs=3, seq_offsets=4096, weight=4096,
                    bias=None, workspace=4096, workspace_bytes=1 << 40)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def scan(**kw):
    p = B.SelectiveScan(dtype=B.NUGPR_FLOAT32, dim=64, groups=2, dim_state=16, softplus=1, n_rows=1000, n_seqs=3,
                        seq_offsets=4096, A=4096, D=None, dt_bias=None, workspace=4096, workspace_bytes=1 << 40)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def conv_calls(lib, p, x=OK, y=OK, s0=None, s1=None):  # noqa: F811
    f, b = lib.nugpr_short_conv_forward, lib.nugpr_short_conv_backward
    yield f(C.byref(p), x, s0, y, s1, None)
    yield b(C.byref(p), x, None, y, s0, y, 4096, 4096, s1, None)


def scan_calls(lib, p, x=OK, b=H, z=None, y=OK, s0=None, s1=None):  # noqa: F811
    yield lib.nugpr_selective_scan_forward(C.byref(p), x, x, b, b, z, s0, y, s1, None)
    yield lib.nugpr_selective_scan_backward(C.byref(p), x, x, b, b, z, None, y, s0, y, y, b, b, z, 4096, 4096, 4096, s1, None)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(dim=0), dict(dim=65537), dict(width=0), dict(width=9), dict(n_rows=-1),
                                dict(n_seqs=-1), dict(n_rows=(1 << 40) + 1)], ids=str)
def test_bad_convolutions(lib, kw):  # noqa: F811
    p = conv(**kw)
    assert lib.nugpr_short_conv_workspace_bytes(C.byref(p)) == 0
    assert list(conv_calls(lib, p)) == [INVALID, INVALID]
    assert lib.nugpr_short_conv_step(C.byref(p), OK, 4096, None, OK, None) == INVALID


def test_bad_calls_of_convolutions(lib):  # noqa: F811
    for bad in (NULL, ODD, BACK, None):
        assert list(conv_calls(lib, conv(), x=bad)) == [INVALID, INVALID]
        assert list(conv_calls(lib, conv(), y=bad)) == [INVALID, INVALID]
    for kw in (dict(weight=None), dict(weight=4097), dict(bias=4098), dict(seq_offsets=None)):
        assert list(conv_calls(lib, conv(**kw))) == [INVALID, INVALID]
    size = 3 * 3 * 64 * 4
    for apart in (0, size - 4):
        assert list(conv_calls(lib, conv(), s0=1 << 20, s1=(1 << 20) + apart)) == [INVALID, INVALID]
        assert list(conv_calls(lib, conv(), s0=(1 << 20) + apart, s1=1 << 20)) == [INVALID, INVALID]
        assert b"overlaps" in lib.nugpr_last_error_string()
    for kw in (dict(workspace=None), dict(workspace=4097), dict(workspace_bytes=10)):
        assert list(conv_calls(lib, conv(**kw)))[1] == WORKSPACE
    b = lib.nugpr_short_conv_backward
    assert b(C.byref(conv()), OK, None, OK, None, OK, None, None, None, None) == INVALID              # nowhere for dweight
    assert b(C.byref(conv(bias=4096)), OK, None, OK, None, OK, 4096, None, None, None) == INVALID     # nor for dbias
    step = lib.nugpr_short_conv_step
    assert step(C.byref(conv()), OK, 4096, None, OK, None) == INVALID                                 # 1000 requests, 3 windows
    assert step(C.byref(conv(n_rows=2)), OK, None, None, OK, None) == INVALID
    assert step(C.byref(conv(n_rows=2)), OK, 4097, None, OK, None) == INVALID
    assert step(C.byref(conv(n_rows=0)), None, None, None, None, None) == B.NUGPR_OK
    assert lib.nugpr_short_conv_forward(C.byref(conv(n_rows=0, n_seqs=0)), None, None, None, None, None) == B.NUGPR_OK


def test_convolutions_beyond_a_launch(lib):  # noqa: F811
    """2^32 threads of one launch: rows there may be as many as there are, windows that are written not."""
    p = conv(n_seqs=1 << 30, dim=65536, workspace_bytes=1 << 62)
    assert list(conv_calls(lib, p, s1=1 << 20)) == [INVALID, INVALID]
    assert b"too many" in lib.nugpr_last_error_string()
    p = conv(n_rows=1 << 30, n_seqs=1 << 30, dim=65536)
    assert lib.nugpr_short_conv_step(C.byref(p), OK, 4096, None, OK, None) == INVALID


@pytest.mark.parametrize("kw", [dict(dtype=-1), dict(dim=0), dict(dim=65538), dict(groups=0), dict(groups=3), dict(groups=128),
                                dict(dim_state=0), dict(dim_state=65), dict(n_rows=-1), dict(n_seqs=-1)], ids=str)
def test_bad_scans(lib, kw):  # noqa: F811
    p = scan(**kw)
    assert lib.nugpr_selective_scan_workspace_bytes(C.byref(p), 0) == 0
    assert len(lib.nugpr_last_error_string()) > 0
    assert list(scan_calls(lib, p)) == [INVALID, INVALID]
    assert lib.nugpr_selective_scan_step(C.byref(p), OK, OK, H, H, None, 4096, None, OK, None) == INVALID


def test_bad_calls_of_scans(lib):  # noqa: F811
    for bad in (NULL, ODD, BACK, None):
        assert list(scan_calls(lib, scan(), x=bad)) == [INVALID, INVALID]
        assert list(scan_calls(lib, scan(), y=bad)) == [INVALID, INVALID]
    for bad in (NULL, ODD, BACK):
        assert list(scan_calls(lib, scan(), z=bad)) == [INVALID, INVALID]
    for bad in (None, B.Heads(None, 1, 1), B.Heads(4096, -1, 1), B.Heads(4096, 1, -1), B.Heads(4098, 1, 1)):
        assert list(scan_calls(lib, scan(), b=bad)) == [INVALID, INVALID]
    for kw in (dict(A=None), dict(A=4097), dict(D=4098), dict(dt_bias=4097), dict(seq_offsets=None), dict(n_seqs=0)):
        assert list(scan_calls(lib, scan(**kw))) == [INVALID, INVALID]
    size = 3 * 64 * 16 * 4
    for apart in (4, size - 4):
        assert list(scan_calls(lib, scan(), s0=1 << 20, s1=(1 << 20) + apart)) == [INVALID, INVALID]
        assert b"overlaps" in lib.nugpr_last_error_string()
    back = lib.nugpr_selective_scan_backward
    assert back(C.byref(scan()), OK, OK, H, H, None, None, OK, 1 << 20, OK, OK, H, H, None, 4096, 4096, 4096, 1 << 20, None) == INVALID
    for kw in (dict(workspace=None), dict(workspace=4097), dict(workspace_bytes=10)):
        assert list(scan_calls(lib, scan(n_rows=1 << 20, **kw))) == [WORKSPACE, WORKSPACE]
    b = lib.nugpr_selective_scan_backward
    for p, sums in ((scan(), (None, 4096, 4096)), (scan(D=4096), (4096, None, 4096)), (scan(dt_bias=4096), (4096, 4096, None))):
        assert b(C.byref(p), OK, OK, H, H, None, None, OK, None, OK, OK, H, H, None, *sums, None, None) == INVALID
    assert b(C.byref(scan()), OK, OK, H, H, OK, None, OK, None, OK, OK, H, H, None, 4096, 4096, 4096, None, None) == INVALID  # no dz
    step = lib.nugpr_selective_scan_step
    assert step(C.byref(scan()), OK, OK, H, H, None, 4096, None, OK, None) == INVALID                 # 1000 requests, 3 states
    assert step(C.byref(scan(n_rows=2)), OK, OK, H, H, None, None, None, OK, None) == INVALID
    assert step(C.byref(scan(n_rows=2)), OK, OK, H, H, None, 4097, None, OK, None) == INVALID
    assert step(C.byref(scan(n_rows=0)), None, None, None, None, None, None, None, None, None) == B.NUGPR_OK
    p = scan(n_rows=0, n_seqs=0)
    assert lib.nugpr_selective_scan_forward(C.byref(p), None, None, None, None, None, None, None, None, None) == B.NUGPR_OK


def test_scans_beyond_a_launch(lib):  # noqa: F811
    p = scan(n_seqs=1 << 27, n_rows=1 << 20, workspace_bytes=1 << 62)
    assert list(scan_calls(lib, p)) == [INVALID, INVALID]
    assert b"too many" in lib.nugpr_last_error_string()
    for rows in (1 << 27, 1 << 40):         # (gradients of B and C: a thread for each of their values)
        p = scan(n_rows=rows, groups=1, workspace_bytes=1 << 62)
        assert lib.nugpr_selective_scan_backward(C.byref(p), OK, OK, H, H, None, None, OK, None, OK, OK, H, H, None, 4096, None,
                                                 None, None, None) == INVALID
        assert b"too many" in lib.nugpr_last_error_string()
    p = scan(n_rows=1 << 30, n_seqs=1 << 30, dim=4096)
    assert lib.nugpr_selective_scan_step(C.byref(p), OK, OK, H, H, None, 4096, None, OK, None) == INVALID


def gradients(*rows):
    return (B.Gradient * len(rows))(*rows)


def test_bad_gradients(lib):  # noqa: F811
    size, norm, clip = lib.nugpr_gradient_norm_workspace_bytes, lib.nugpr_gradient_norm, lib.nugpr_clip_gradients

    def calls(g, to=4096, ws=4096, ws_bytes=1 << 30, bound=1.0):
        return [norm(g, len(g), to, ws, ws_bytes, None), clip(g, len(g), bound, to, ws, ws_bytes, None)]

    for bad in ((4096, None, 10, 2, 0), (4096, None, -1, 0, 0), (4096, None, (1 << 40) + 1, 0, 0)):
        g = gradients((4096, None, 5, 0, 0), bad)
        assert size(g, 2) == 0 and calls(g) == [INVALID, INVALID]
    for bad in ((None, None, 10, 0, 0), (4098, None, 10, 0, 0), (4097, None, 10, 1, 0)):
        assert calls(gradients(bad)) == [INVALID, INVALID]
    g = gradients((4096, None, 10, 0, 0))
    assert calls(g, to=None) == [INVALID, INVALID] and calls(g, to=4097) == [INVALID, INVALID]
    assert calls(g, ws=None) == [WORKSPACE, WORKSPACE] and calls(g, ws=4097) == [WORKSPACE, WORKSPACE]
    assert calls(g, ws_bytes=8) == [WORKSPACE, WORKSPACE]
    for bound in (-1.0, float("nan")):
        assert calls(g, bound=bound)[1] == INVALID
    for bad in ((4096, 8192, 10, 0, 3), (4096, 8194, 10, 0, 0), (4096, 4100, 10, 0, 0), (4096, 4096, 10, 0, 1)):
        assert calls(gradients(bad))[1] == INVALID
    for two in (((4096, None, 10, 0, 0), (4132, None, 5, 1, 0)), ((4096, 8192, 10, 0, 0), (4200, 8230, 5, 1, 1)),
                ((4096, 8192, 10, 0, 0), (8230, 16384, 5, 1, 1)), ((1 << 20, 8192, 1000, 1, 1), (8400, None, 5, 0, 0))):
        for order in (two, two[::-1]):
            assert calls(gradients(*order))[1] == INVALID
            assert b"overlap" in lib.nugpr_last_error_string()
    assert size(None, 1) == 0 and size(g, -1) == 0 and size(None, 0) > 0
    many = gradients(*[(4096, None, 1 << 20, 0, 0)] * 3000)
    assert 256 < size(many, 3000) < 64 * 1024                    # a few thousand partial sums, however many tensors
