"""Offsets that do not ascend or lie outside the rows (GPU): whatever the results are, memory around the outputs stays as it is."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2510_12128_amd import binding as B

pytestmark = pytest.mark.gpu

GUARD = 4096            # rows beside an array on either side
MARK = 77.0


class Guarded:
    """Rows x heads x width in the middle of a larger array of MARK."""

    def __init__(self, n, heads, width, dtype, fill=True):
        self.all = torch.full((n + 2 * GUARD, heads, width), MARK, dtype=dtype, device="cuda")
        self.rows = self.all[GUARD:GUARD + n]
        if fill:
            self.rows.copy_(torch.randn(n, heads, width, generator=torch.Generator().manual_seed(n + width)).to(dtype))
        self.heads = C.byref(B.Heads(self.rows.data_ptr(), heads * width, width))

    def untouched(self):
        return bool((self.all[:GUARD] == MARK).all() and (self.all[-GUARD:] == MARK).all())


def bad_offsets(n):
    rng = np.random.default_rng(n)
    yield [n // 2 + 70, 10, n - 7, n]
    yield [n, 0]
    yield [n - 1, n - 2, 5, 3, 1]
    yield [-10 ** 12, 10 ** 12, -5, n + 5]
    for count in (3, 9, 200):
        yield rng.integers(-50, n + 50, size=count).tolist()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 300, 1500])
def test_memory_around_the_outputs_stays(lib, n, dtype):
    c, h, kv, dk, dv = B.load_library(), 4, 2, 64, 40
    z = B.NUGPR_FLOAT32 if dtype == torch.float32 else B.NUGPR_BFLOAT16
    g = torch.full((kv,), -0.01, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    for off in bad_offsets(n):
        dev = torch.tensor(off, dtype=torch.int64, device="cuda")
        q, k, v, do = (Guarded(n, x, w, dtype) for x, w in ((h, dk), (kv, dk), (kv, dv), (h, dv)))
        o, dq, dk_, dv_ = (Guarded(n, x, w, dtype, False) for x, w in ((h, dv), (h, dk), (kv, dk), (kv, dv)))
        p = B.DecayAttention(z, h, kv, dk, dv, n, len(off) - 1, dev.data_ptr(), g.data_ptr(), 1.0, None, 0)
        for backward in (0, 1):
            need = c.nugpr_decay_attention_workspace_bytes(C.byref(p), backward)
            ws = torch.empty(need, dtype=torch.uint8, device="cuda")
            p.workspace, p.workspace_bytes = ws.data_ptr(), need
            if backward:
                code = c.nugpr_decay_attention_backward(C.byref(p), q.heads, k.heads, v.heads, None, do.heads, None, dq.heads, dk_.heads, dv_.heads, None, stream)
            else:
                code = c.nugpr_decay_attention_forward(C.byref(p), q.heads, k.heads, v.heads, None, o.heads, None, stream)
            assert code == B.NUGPR_OK
            torch.cuda.synchronize()
        assert all(x.untouched() for x in (o, dq, dk_, dv_)), off
        x, dy = Guarded(n, 1, 96, dtype), Guarded(n, 1, 72, dtype)
        y, dx = Guarded(n, 1, 72, dtype, False), Guarded(n, 1, 96, dtype, False)
        W, A, Bs = (torch.randn(*s, device="cuda").to(dtype) for s in ((72, 96), (3, 8, 96), (3, 8, 72)))
        dA, dB = torch.empty_like(A), torch.empty_like(Bs)
        which = (torch.arange(len(off) - 1, device="cuda") % 3).int()
        p = B.Adapter(z, 96, 72, 8, 3, n, len(off) - 1, dev.data_ptr(), which.data_ptr(), W.data_ptr(), A.data_ptr(), Bs.data_ptr(), 1.0, None, 0)
        need = c.nugpr_adapter_workspace_bytes(C.byref(p), 1)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        p.workspace, p.workspace_bytes = ws.data_ptr(), need
        assert c.nugpr_adapter_forward(C.byref(p), x.rows.data_ptr(), 96, y.rows.data_ptr(), stream) == B.NUGPR_OK
        assert c.nugpr_adapter_backward(C.byref(p), x.rows.data_ptr(), 96, dy.rows.data_ptr(), 72, dx.rows.data_ptr(), dA.data_ptr(),
                                        dB.data_ptr(), stream) == B.NUGPR_OK
        torch.cuda.synchronize()
        assert y.untouched() and dx.untouched(), off
