"""How the convolution, the scan and the clipping are called (GPU): autograd, graphs, streams, offsets that lie, arrays beyond
32 bits, the same results each time."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2510_12128_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def conv(n=90, dim=70, width=4, dtype=F32, seed=0, seqs=(0, 40, 40, 90)):
    gen = torch.Generator().manual_seed(seed)

    def r(*shape, t=dtype):
        return torch.randn(*shape, generator=gen).to(t).cuda()

    k = len(seqs) - 1
    return (dict(x=r(n, dim), weight=r(dim, width), seq_offsets=torch.tensor(seqs, device="cuda"), bias=r(dim), silu=True,
                 initial_state=r(k, width - 1, dim)),
            dict(d_y=r(n, dim), d_final_state=r(k, width - 1, dim)))


def scan(n=90, dim=70, states=16, dtype=F32, seed=0, seqs=(0, 40, 40, 90)):
    gen = torch.Generator().manual_seed(seed)

    def r(*shape, t=dtype):
        return torch.randn(*shape, generator=gen).to(t).cuda()

    k = len(seqs) - 1
    return (dict(x=r(n, dim), dt=r(n, dim) - 2.0, A=-torch.rand(dim, states, generator=gen).cuda() - 0.1, B=r(n, 1, states), C=r(n, 1, states),
                 seq_offsets=torch.tensor(seqs, device="cuda"), D=r(dim, t=F32), z=r(n, dim), dt_bias=r(dim, t=F32),
                 initial_state=r(k, dim, states, t=F32)),
            dict(d_y=r(n, dim), d_final_state=r(k, dim, states, t=F32)))


def as_step(args, rows):
    one = {k: t[:rows] if k in ("x", "dt", "B", "C", "z") else t for k, t in args.items() if k not in ("seq_offsets", "initial_state")}
    return dict(one, state=args["initial_state"].clone())


def calls(lib):
    a, g = conv()
    yield lib.nugpr_short_conv_forward, a
    yield lib.nugpr_short_conv_backward, dict(a, **g)
    yield lib.nugpr_short_conv_step, as_step(a, 3)
    a, g = scan()
    yield lib.nugpr_selective_scan_forward, a
    yield lib.nugpr_selective_scan_backward, dict(a, **g)
    yield lib.nugpr_selective_scan_step, as_step(a, 3)


def test_inputs_that_require_gradients_are_refused(lib):
    for call, args in calls(lib):
        for name, t in args.items():
            if not isinstance(t, torch.Tensor) or not t.is_floating_point():
                continue
            given = dict(args, **{name: t.detach().clone().requires_grad_()})
            with pytest.raises(lib.NugprError, match=f"{name} requires a gradient"):
                call(**given)
            with torch.no_grad():
                call(**given)


def test_a_step_says_that_it_has_written_the_state(lib):
    for call, args in calls(lib):
        if "state" in args:
            before = args["state"]._version
            call(**args)
            assert args["state"]._version == before + 1


def test_arguments_that_do_not_fit_are_refused(lib):
    for call, args in calls(lib):
        for name, t in args.items():
            if not isinstance(t, torch.Tensor):
                continue
            bad = [t.cpu(), t.double() if t.is_floating_point() else t.int(), t[..., None]]
            if name != "seq_offsets" and t.numel() > 1:
                bad.append(torch.cat([t, t], dim=-1))
                if t.dim() > 1:
                    bad.append(torch.stack([t, t], dim=-1)[..., 0])     # (the last dimension is not contiguous)
            for b in bad:
                with pytest.raises(lib.NugprError):
                    call(**dict(args, **{name: b}))


def flat(out):
    return [t for t in (out if isinstance(out, tuple) else (out,)) if t is not None]


def test_the_same_twice(lib):
    for dtype in (F32, BF16):
        for (a, g), f, b in ((conv(3000, 130, dtype=dtype, seqs=(0, 1000, 1001, 3000)), lib.nugpr_short_conv_forward, lib.nugpr_short_conv_backward),
                             (scan(3000, 130, dtype=dtype, seqs=(0, 1000, 1001, 3000)), lib.nugpr_selective_scan_forward, lib.nugpr_selective_scan_backward)):
            first = flat(f(**a)) + flat(b(**a, **g))
            for _ in range(3):
                for x, y in zip(flat(f(**a)) + flat(b(**a, **g)), first):
                    assert torch.equal(x, y)


def test_graphs_replay(lib):
    """Two graphs of the same calls, replayed in turn on new inputs, with eager calls between: every replay is the eager result."""
    args = [conv(300, seqs=(0, 200, 300), dtype=BF16), scan(300, seqs=(0, 200, 300), dtype=BF16)]
    grads = [torch.randn(5000, device="cuda"), torch.randn(77, device="cuda").to(BF16)]
    out = [torch.empty_like(t) for t in grads]

    def run(states):
        r = []
        for (a, g), f, b, s, st in zip(args, (lib.nugpr_short_conv_forward, lib.nugpr_selective_scan_forward),
                                       (lib.nugpr_short_conv_backward, lib.nugpr_selective_scan_backward),
                                       (lib.nugpr_short_conv_step, lib.nugpr_selective_scan_step), states):
            r += flat(f(**a)) + flat(b(**a, **g)) + flat(s(**dict(as_step(a, 2), state=st)))
        return r + [lib.nugpr_gradient_norm(grads), lib.nugpr_clip_gradients(grads, 3.0, out=out)]

    def fresh():
        return [a["initial_state"].clone() for a, _ in args]

    run(fresh())
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        states, graph = fresh(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = run(states)
        graphs.append((graph, states, got))
    for r in range(3):
        for graph, states, got in graphs:
            for (a, g) in args:
                a["x"].copy_(torch.randn(a["x"].shape, device="cuda"))
                g["d_y"].copy_(torch.randn(g["d_y"].shape, device="cuda"))
            for t in grads:
                t.copy_(torch.randn(t.shape, device="cuda"))
            for s, (a, _) in zip(states, args):
                s.copy_(a["initial_state"])
            eager_states = fresh()
            want = run(eager_states) + [t.clone() for t in out]
            graph.replay()
            torch.cuda.synchronize()
            for x, y in zip(got + out, want):
                assert torch.equal(x, y)
            for x, y in zip(states, eager_states):
                assert torch.equal(x, y)


def test_two_streams_at_once(lib):
    sets = [scan(2000, 200, seed=s, seqs=(0, 1500, 2000)) for s in (1, 2)]
    want = [flat(lib.nugpr_selective_scan_forward(**a)) + flat(lib.nugpr_selective_scan_backward(**a, **g)) for a, g in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(3):
        for i, ((a, g), s) in enumerate(zip(sets, streams)):
            with torch.cuda.stream(s):
                got[i] = flat(lib.nugpr_selective_scan_forward(**a)) + flat(lib.nugpr_selective_scan_backward(**a, **g))
    torch.cuda.synchronize()
    for x, y in zip(got[0] + got[1], want[0] + want[1]):
        assert torch.equal(x, y)


def test_end_states_may_be_written_over_the_start_states(lib):
    """Through the C entry point: sequences of no span, of one and of many."""
    a, _ = scan(3030, 80, dtype=BF16, seqs=(0, 0, 30, 3030))
    want_y, want_s = lib.nugpr_selective_scan_forward(**a)
    c, y, s = B.load_library(), torch.empty_like(want_y), a["initial_state"].clone()
    p = B.SelectiveScan(B.NUGPR_BFLOAT16, 80, 1, 16, 1, 3030, 3, a["seq_offsets"].data_ptr(), a["A"].data_ptr(), a["D"].data_ptr(),
                        a["dt_bias"].data_ptr(), None, 0)
    need = c.nugpr_selective_scan_workspace_bytes(C.byref(p), 0)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    p.workspace, p.workspace_bytes = ws.data_ptr(), need
    x, dt, z, out = (C.byref(B.Rows(t.data_ptr(), 80)) for t in (a["x"], a["dt"], a["z"], y))
    b, cc = (C.byref(B.Heads(t.data_ptr(), 16, 16)) for t in (a["B"], a["C"]))
    assert c.nugpr_selective_scan_forward(C.byref(p), x, dt, b, cc, z, s.data_ptr(), out, s.data_ptr(),
                                          torch.cuda.current_stream().cuda_stream) == B.NUGPR_OK
    assert torch.equal(y, want_y) and torch.equal(s, want_s)


GUARD, MARK = 4096, 77.0           # rows beside an array on either side


class Guarded:
    """Rows x width in the middle of a larger array of MARK."""

    def __init__(self, n, width, dtype, fill=True):
        self.all = torch.full((n + 2 * GUARD, width), MARK, dtype=dtype, device="cuda")
        self.rows = self.all[GUARD:GUARD + n]
        if fill:
            self.rows.copy_(torch.randn(n, width, generator=torch.Generator().manual_seed(n + width)).to(dtype))
        self.array, self.heads = C.byref(B.Rows(self.rows.data_ptr(), width)), C.byref(B.Heads(self.rows.data_ptr(), width, width))

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


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [1, 300, 1500])
def test_offsets_that_lie_leave_the_memory_around_the_outputs(lib, n, dtype):
    c, dim, width, states, t = B.load_library(), 72, 4, 16, B.NUGPR_FLOAT32 if dtype == F32 else B.NUGPR_BFLOAT16
    stream = torch.cuda.current_stream().cuda_stream

    def workspace(p, need):
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        p.workspace, p.workspace_bytes = ws.data_ptr(), need
        return ws

    for off in bad_offsets(n):
        dev, k = torch.tensor(off, dtype=torch.int64, device="cuda"), len(off) - 1
        x, dy, dt, z, y, dx, ddt, dz = (Guarded(n, dim, dtype, i < 4) for i in range(8))
        b, cc, db, dc = (Guarded(n, states, dtype, i < 2) for i in range(4))
        # sums and states, in rows of one sequence (or one channel) each
        w0, w1, dw0 = (Guarded(k, (width - 1) * dim, dtype) for _ in range(3))
        s0, s1, ds0 = (Guarded(k, dim * states, F32) for _ in range(3))
        dweight, dA, sums = Guarded(dim, width, dtype), Guarded(dim, states, F32), Guarded(dim, 1, F32)
        weight, A = torch.randn(dim, width, device="cuda").to(dtype), -torch.rand(dim, states, device="cuda")
        vec = torch.randn(dim, device="cuda")
        p = B.ShortConv(t, dim, width, 1, n, k, dev.data_ptr(), weight.data_ptr(), None, None, 0)
        ws = workspace(p, c.nugpr_short_conv_workspace_bytes(C.byref(p)))
        assert c.nugpr_short_conv_forward(C.byref(p), x.array, w0.rows.data_ptr(), y.array, w1.rows.data_ptr(), stream) == B.NUGPR_OK
        assert c.nugpr_short_conv_backward(C.byref(p), x.array, w0.rows.data_ptr(), dy.array, w1.rows.data_ptr(), dx.array,
                                           dweight.rows.data_ptr(), None, dw0.rows.data_ptr(), stream) == B.NUGPR_OK
        torch.cuda.synchronize()
        p = B.SelectiveScan(t, dim, 1, states, 1, n, k, dev.data_ptr(), A.data_ptr(), vec.data_ptr(), None, None, 0)
        ws = workspace(p, c.nugpr_selective_scan_workspace_bytes(C.byref(p), 0))
        assert c.nugpr_selective_scan_forward(C.byref(p), x.array, dt.array, b.heads, cc.heads, z.array, s0.rows.data_ptr(), y.array,
                                              s1.rows.data_ptr(), stream) == B.NUGPR_OK
        torch.cuda.synchronize()
        ws = workspace(p, c.nugpr_selective_scan_workspace_bytes(C.byref(p), 1))  # noqa: F841
        assert c.nugpr_selective_scan_backward(C.byref(p), x.array, dt.array, b.heads, cc.heads, z.array, s0.rows.data_ptr(), dy.array,
                                               s1.rows.data_ptr(), dx.array, ddt.array, db.heads, dc.heads, dz.array, dA.rows.data_ptr(),
                                               sums.rows.data_ptr(), None, ds0.rows.data_ptr(), stream) == B.NUGPR_OK
        torch.cuda.synchronize()
        for a in (x, dy, dt, z, y, dx, ddt, dz, b, cc, db, dc, w0, w1, dw0, s0, s1, ds0, dweight, dA, sums):
            assert a.untouched(), off


def test_arrays_beyond_32_bits(lib):
    """Rows 2^31 values apart and more, and a state that begins beyond 2^32 bytes."""
    step = (1 << 31) + 24
    big = torch.empty(2 * step + 64, dtype=BF16, device="cuda")
    far = big.as_strided((3, 64), (step, 1))
    near = torch.randn(3, 64, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    far.copy_(near)
    a, g = conv(3, 64, dtype=BF16, seqs=(0, 2, 3))
    for x, y in zip(flat(lib.nugpr_short_conv_forward(**dict(a, x=far))), flat(lib.nugpr_short_conv_forward(**dict(a, x=near)))):
        assert torch.equal(x, y)
    for x, y in zip(flat(lib.nugpr_short_conv_backward(**dict(a, x=far), **dict(g, d_y=far))),
                    flat(lib.nugpr_short_conv_backward(**dict(a, x=near), **dict(g, d_y=near)))):
        assert torch.equal(x, y)
    a, g = scan(3, 64, dtype=BF16, seqs=(0, 2, 3))
    for x, y in zip(flat(lib.nugpr_selective_scan_forward(**dict(a, x=far, z=far))), flat(lib.nugpr_selective_scan_forward(**dict(a, x=near, z=near)))):
        assert torch.equal(x, y)
    for x, y in zip(flat(lib.nugpr_selective_scan_backward(**dict(a, x=far, dt=far), **dict(g, d_y=far))),
                    flat(lib.nugpr_selective_scan_backward(**dict(a, x=near, dt=near), **dict(g, d_y=near)))):
        assert torch.equal(x, y)
    del big, far
    a, _ = scan(2, 1024, states=64, seqs=(0, 1, 2))
    pool = torch.empty(20000, 1024, 64, device="cuda")           # 5 GiB
    slots = torch.tensor([19999, 17000], dtype=torch.int32, device="cuda")
    small = as_step(a, 2)
    pool[slots.long()] = small["state"]
    y = lib.nugpr_selective_scan_step(**dict(small, state=pool, slots=slots))
    assert torch.equal(y, lib.nugpr_selective_scan_step(**small)) and torch.equal(pool[slots.long()], small["state"])


def test_the_longest_sequence_of_many(lib):
    """Sequences and rows in the thousands: all short but one."""
    lens = [1] * 3000 + [0] * 50 + [5000] + [2] * 1000
    off = np.concatenate([[0], np.cumsum(lens)]).tolist()
    a, g = scan(off[-1], 64, states=4, seqs=off)
    y, end = lib.nugpr_selective_scan_forward(**a)
    alone = {k: t[3000:8000] if k in ("x", "dt", "B", "C", "z") else t for k, t in a.items()}
    w, w_end = lib.nugpr_selective_scan_forward(**dict(alone, seq_offsets=torch.tensor([0, 5000], device="cuda"),
                                                       initial_state=a["initial_state"][3050:3051]))
    # (spans of another length: the same sums in another order)
    assert float((y[3000:8000] - w).norm()) <= 64 * 2.0 ** -24 * float(w.norm())
    assert float((end[3050:3051] - w_end).norm()) <= 64 * 2.0 ** -24 * float(w_end.norm())
    d = lib.nugpr_selective_scan_backward(**a, **g)
    assert all(bool(torch.isfinite(t).all()) for t in d)
    a, g = conv(off[-1], 64, seqs=off)
    y, end = lib.nugpr_short_conv_forward(**a)
    w, w_end = lib.nugpr_short_conv_forward(**dict(a, x=a["x"][3000:8000], seq_offsets=torch.tensor([0, 5000], device="cuda"),
                                                   initial_state=a["initial_state"][3050:3051]))
    assert torch.equal(y[3000:8000], w) and torch.equal(end[3050:3051], w_end)
    assert all(bool(torch.isfinite(t).all()) for t in lib.nugpr_short_conv_backward(**a, **g))
