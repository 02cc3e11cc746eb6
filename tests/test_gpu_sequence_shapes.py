"""Shapes and strides of the sequence operators (GPU) that a packed batch has beside the plain ones: hundreds of sequences or
requests, slices of one buffer, arrays that repeat one row or head, rows that no sequence owns.  References and tolerances of
tests/test_gpu_decay_attention.py and tests/test_gpu_adapter.py."""
import ctypes as C

import numpy as np
import pytest
import torch

import test_gpu_adapter as adapters
import test_gpu_decay_attention as attention
from paper_2510_12128_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("count", [65, 200, 4200])
def test_many_sequences(lib, count, dtype):
    """One round, two and three of the search for a workgroup's sequence."""
    rng = np.random.default_rng(count)
    lens = rng.integers(0, 4 if count > 1000 else 9, size=count).tolist()
    lens[count // 2] = 300
    q, k, v, do, g, off, dev_off, S0, dS1 = attention.inputs(lens, 2, 1, 16, 24, dtype, seed=count)
    o, S = lib.nugpr_decay_attention_forward(q, k, v, g, dev_off, scale=0.5, initial_state=S0)
    want, end = attention.reference(q, k, v, g, off, 0.5, S0)
    attention.close(o, want, attention.TOL[dtype])
    attention.close(S, end, attention.TOL[F32])
    got = lib.nugpr_decay_attention_backward(q, k, v, g, dev_off, do, scale=0.5, initial_state=S0, d_final_state=dS1)
    for x, w, name in zip(got, attention.reference_backward(q, k, v, g, off, 0.5, do, S0, dS1), ("dq", "dk", "dv", "dS")):
        attention.close(x, w, attention.TOL[F32] if name == "dS" else attention.TOL[dtype], name)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [64, 40, 33])
def test_slices_of_one_buffer(lib, width, dtype):
    lens = [70, 3, 130]
    n, h, kv = sum(lens), 4, 2
    every = torch.randn(n, h + 2 * kv, width, generator=torch.Generator().manual_seed(width)).to(dtype).cuda()
    q, k, v = every[:, :h], every[:, h:h + kv], every[:, h + kv:]
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    g, dev_off = torch.tensor([-0.1, -0.01], device="cuda"), torch.from_numpy(off).cuda()
    o, S = lib.nugpr_decay_attention_forward(q, k, v, g, dev_off)
    want, end = attention.reference(q, k, v, g, off, 1.0)
    attention.close(o, want, attention.TOL[dtype])
    attention.close(S, end, attention.TOL[F32])
    do, zero = torch.randn(n, h, width, device="cuda").to(dtype), torch.zeros_like(S)
    got = lib.nugpr_decay_attention_backward(q, k, v, g, dev_off, do)
    for x, w, name in zip(got, attention.reference_backward(q, k, v, g, off, 1.0, do, zero, zero), ("dq", "dk", "dv", "dS")):
        attention.close(x, w, attention.TOL[F32] if name == "dS" else attention.TOL[dtype], name)
    state = torch.randn(n, kv, width, width, device="cuda")
    kept = state.clone()
    one = torch.arange(n + 1).numpy()
    want, end = attention.reference(q, k, v, g, one, 1.0, kept)
    attention.close(lib.nugpr_decay_attention_step(q, k, v, g, state), want, attention.TOL[dtype])
    attention.close(state, end, attention.TOL[F32])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("over", ["heads", "rows", "both"])
def test_arrays_that_repeat_a_row_or_a_head(lib, over, dtype):
    lens, width = [70, 3, 130], 48
    n, h, kv = sum(lens), 4, 2
    gen = torch.Generator().manual_seed(5)

    def r(heads):
        shape = {"heads": (n, 1, width), "rows": (1, heads, width), "both": (1, 1, width)}[over]
        return torch.randn(*shape, generator=gen).to(dtype).cuda().expand(n, heads, width)

    q, k, v, do = r(h), r(kv), r(kv), r(h)
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    g, dev_off = torch.tensor([-0.1, -0.01], device="cuda"), torch.from_numpy(off).cuda()
    o, S = lib.nugpr_decay_attention_forward(q, k, v, g, dev_off, scale=0.2)
    want, end = attention.reference(q, k, v, g, off, 0.2)
    attention.close(o, want, attention.TOL[dtype])
    attention.close(S, end, attention.TOL[F32])
    zero = torch.zeros_like(S)
    got = lib.nugpr_decay_attention_backward(q, k, v, g, dev_off, do, scale=0.2)
    for x, w, name in zip(got, attention.reference_backward(q, k, v, g, off, 0.2, do, zero, zero), ("dq", "dk", "dv", "dS")):
        attention.close(x, w, attention.TOL[F32] if name == "dS" else attention.TOL[dtype], name)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dk,dv", [(64, 64), (24, 17), (128, 128)])
def test_rows_without_a_sequence_are_written(lib, dk, dv, dtype):
    """Outputs that held NaN before: zero outside the sequences, and no NaN left inside."""
    c, n, h, kv = B.load_library(), 700, 4, 2
    q, k, v, do, g, _, _, _, _ = attention.inputs([n], h, kv, dk, dv, dtype, seed=7)
    off = np.array([20, 90, 90, 500])
    dev = torch.from_numpy(off).cuda()
    stream = torch.cuda.current_stream().cuda_stream
    o, dq, dk_, dv_ = (torch.full(x.shape, float("nan"), dtype=dtype, device="cuda") for x in (do, q, k, v))
    p = B.DecayAttention(B.NUGPR_FLOAT32 if dtype == F32 else B.NUGPR_BFLOAT16, h, kv, dk, dv, n, 3, dev.data_ptr(), g.data_ptr(), 1.0, None, 0)
    heads = [C.byref(B.Heads(x.data_ptr(), x.stride(0), x.stride(1))) for x in (q, k, v, do, o, dq, dk_, dv_)]
    need = max(c.nugpr_decay_attention_workspace_bytes(C.byref(p), b) for b in (0, 1))
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")                    # (NaN, too)
    p.workspace, p.workspace_bytes = ws.data_ptr(), need
    assert c.nugpr_decay_attention_forward(C.byref(p), *heads[:3], None, heads[4], None, stream) == B.NUGPR_OK
    assert c.nugpr_decay_attention_backward(C.byref(p), *heads[:3], None, heads[3], None, *heads[5:], None, stream) == B.NUGPR_OK
    for x in (o, dq, dk_, dv_):
        assert not x[:20].any() and not x[500:].any() and torch.isfinite(x).all()
    want, _ = attention.reference(q, k, v, g, off, 1.0)
    attention.close(o, want, attention.TOL[dtype])


def on_gpu(x, W, A, B, off, which, scale, dy):
    """The adapters' reference in float64 on the GPU, request by request."""
    x, W, A, B, dy = (t.double() for t in (x, W, A, B, dy))
    y, dx, dA, dB = x @ W.T, dy @ W, torch.zeros_like(A), torch.zeros_like(B)
    for s, a in enumerate(which):
        r = slice(int(off[s]), int(off[s + 1]))
        if 0 <= a < A.shape[0] and off[s + 1] > off[s]:
            low, up = scale * (x[r] @ A[a].T), scale * (dy[r] @ B[a].T)
            y[r] += low @ B[a]
            dx[r] += up @ A[a]
            dA[a] += up.T @ x[r]
            dB[a] += low.T @ dy[r]
    return y, dx, dA, dB


# (requests, rows of one, width in, width out, rank): few columns in one pass; tiles of 128; of 128 and of 256 rows in bfloat16
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("count,each,inp,out,rank", [(1200, 1, 96, 40, 8), (1100, 4, 200, 1000, 20), (1500, 1, 512, 2304, 8), (1024, 4, 128, 4096, 40),
                                                     (600, 9, 2104, 192, 5)])
def test_many_requests_in_every_kind_of_tile(lib, count, each, inp, out, rank, dtype):
    lens = [each + (s % 3 == 0) - (s % 5 == 0) for s in range(count)]
    x, W, A, B_, off, dev_off, _, _, dy = adapters.inputs(lens, inp, out, rank, 7, dtype, seed=count)
    which = [-1 if s % 11 == 3 else s % 7 for s in range(count)]
    dev_which = torch.tensor(which, dtype=torch.int32, device="cuda")
    want = on_gpu(x, W, A, B_, off, which, 1.5, dy)
    got = (lib.nugpr_adapter_forward(x, W, A, B_, dev_off, adapter_of=dev_which, scale=1.5),
           *lib.nugpr_adapter_backward(x, W, A, B_, dev_off, dy, adapter_of=dev_which, scale=1.5))
    for g, w in zip(got, want):
        adapters.close(g, w.cpu(), adapters.TOL[dtype])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("inp,out,rank", [(20, 24, 40), (40, 20, 3), (24, 32, 33), (17, 31, 5)])
def test_many_rows_of_few_columns(lib, inp, out, rank, dtype):
    x, W, A, B_, off, dev_off, which, dev_which, dy = adapters.inputs([20000, 14003], inp, out, rank, 2, dtype, seed=inp)
    want = on_gpu(x, W, A, B_, off, which, 1.0, dy)
    got = (lib.nugpr_adapter_forward(x, W, A, B_, dev_off, adapter_of=dev_which), *lib.nugpr_adapter_backward(x, W, A, B_, dev_off, dy, adapter_of=dev_which))
    for (g, w), name in zip(zip(got, want), ("y", "dx", "dA", "dB")):
        # sums over up to 20000 rows: four times as many roundings as the 4096 of the tolerance, by the square root twice it
        adapters.close(g, w.cpu(), adapters.TOL[dtype] * (2.5 if name in ("dA", "dB") else 1))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_x_that_repeat(lib, dtype):
    x, W, A, B_, off, dev_off, which, dev_which, dy = adapters.inputs([100, 200], 64, 48, 4, 2, dtype, seed=3)
    xs, dys = x[:1].expand(300, 64), dy[:1].expand(300, 48)
    want = on_gpu(xs, W, A, B_, off, which, 1.0, dys)
    got = (lib.nugpr_adapter_forward(xs, W, A, B_, dev_off, adapter_of=dev_which), *lib.nugpr_adapter_backward(xs, W, A, B_, dev_off, dys, adapter_of=dev_which))
    for g, w in zip(got, want):
        adapters.close(g, w.cpu(), adapters.TOL[dtype])
