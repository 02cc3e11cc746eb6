"""Linear attention with decay (GPU) against the recurrence itself in 64 bits, token by token.

Tolerances, relative in the 2-norm.  float32: sums of up to 128 products, of 64 rows of a block and of a state that each of
the blocks rounds once, each rounding 2^-24 and independent of the others: well below 64 of them.  bfloat16 outputs: the
result is rounded once to 8 bits (2^-9) and so are the weights inside a block; two roundings, 2^-8.  States are summed in
float32 from exact products, whatever the inputs' type."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
TOL = {F32: 64 * 2.0 ** -24, BF16: 2.0 ** -8}


def reference(q, k, v, g, offsets, scale, S0=None):
    """o, end states; everything in float64 on the CPU."""
    q, k, v, g = (x.double().cpu() for x in (q, k, v, g))
    n, h, dk = q.shape
    kv, dv = k.shape[1], v.shape[2]
    o = torch.zeros(n, h, dv, dtype=torch.float64)
    ends = []
    for s in range(len(offsets) - 1):
        S = torch.zeros(kv, dk, dv, dtype=torch.float64) if S0 is None else S0[s].double().cpu().clone()
        for t in range(offsets[s], offsets[s + 1]):
            S = torch.exp(g)[:, None, None] * S + k[t][:, :, None] * v[t][:, None, :]
            o[t] = scale * (q[t].reshape(kv, -1, dk) @ S).reshape(h, dv)
        ends.append(S)
    return o, torch.stack(ends)


def reference_backward(q, k, v, g, offsets, scale, do, S0, dS1):
    """By the recurrences S_t and U_t."""
    q, k, v, g, do, S0, dS1 = (x.double().cpu() for x in (q, k, v, g, do, S0, dS1))
    lam = torch.exp(g)[:, None, None]
    kv, dk, dv = k.shape[1], q.shape[2], v.shape[2]
    dq, dk_, dv_, dS = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v), torch.zeros_like(S0)
    for s in range(len(offsets) - 1):
        S = S0[s].clone()
        for t in range(offsets[s], offsets[s + 1]):
            S = lam * S + k[t][:, :, None] * v[t][:, None, :]
            dq[t] = scale * (do[t].reshape(kv, -1, dv) @ S.transpose(1, 2)).reshape(q[t].shape)
        U = dS1[s].clone()
        for t in reversed(range(offsets[s], offsets[s + 1])):
            U = U + scale * q[t].reshape(kv, -1, dk).transpose(1, 2) @ do[t].reshape(kv, -1, dv)
            dk_[t] = (U @ v[t][:, :, None])[:, :, 0]
            dv_[t] = (k[t][:, None, :] @ U)[:, 0]
            U = lam * U
        dS[s] = U
    return dq, dk_, dv_, dS


def close(x, want, tol, what=""):
    assert x.shape == want.shape, what
    x, want = x.double().cpu(), want.double()
    err = float((x - want).norm())
    assert err <= tol * float(want.norm()) or err == 0.0, (what, err / float(want.norm() + 1e-300))


def inputs(lens, h, kv, dk, dv, dtype, seed=0, layout="dense"):
    gen = torch.Generator().manual_seed(seed)
    n = sum(lens)

    def r(*shape):
        return torch.randn(*shape, generator=gen)

    def place(x):
        x = x.to(dtype)
        if layout == "dense":
            return x.cuda()
        if layout == "heads first":                   # heads x rows x width, seen as rows x heads x width
            return x.transpose(0, 1).contiguous().cuda().transpose(0, 1)
        if layout == "odd":                           # rows that begin at any value
            wide = torch.zeros(n, x.shape[1], x.shape[2] + 3, dtype=dtype, device="cuda")
            wide[:, :, 1:1 + x.shape[2]] = x.cuda()
            return wide[:, :, 1:1 + x.shape[2]]
        raise AssertionError(layout)

    q, k, v, do = r(n, h, dk), r(n, kv, dk), r(n, kv, dv), r(n, h, dv)
    g = torch.log1p(-2.0 ** -torch.linspace(1, 10, kv)).cuda()
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    S0, dS1 = r(len(lens), kv, dk, dv).cuda(), r(len(lens), kv, dk, dv).cuda()
    return tuple(place(x) for x in (q, k, v, do)) + (g, off, torch.from_numpy(off).cuda(), S0, dS1)


LENS = [[1], [63], [64], [65], [0, 1, 0, 2, 129, 0], [300, 7, 64, 128, 1], [700]]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("h,kv,dk,dv", [(2, 2, 64, 64), (4, 1, 128, 128), (3, 3, 5, 17), (6, 2, 72, 128)])
def test_forward(lib, lens, h, kv, dk, dv, dtype):
    q, k, v, _, g, off, dev_off, S0, _ = inputs(lens, h, kv, dk, dv, dtype, seed=len(lens) + dk)
    for start in (None, S0):
        o, S = lib.nugpr_decay_attention_forward(q, k, v, g, dev_off, scale=0.3, initial_state=start)
        want, end = reference(q, k, v, g, off, 0.3, start)
        assert o.dtype == dtype and S.dtype == F32
        close(o, want, TOL[dtype], "o")
        close(S, end, TOL[F32], "state")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("h,kv,dk,dv", [(2, 2, 64, 64), (4, 1, 128, 128), (3, 3, 5, 17), (6, 2, 72, 128)])
def test_backward(lib, lens, h, kv, dk, dv, dtype):
    q, k, v, do, g, off, dev_off, S0, dS1 = inputs(lens, h, kv, dk, dv, dtype, seed=3 * len(lens) + dk)
    zero = torch.zeros_like(S0)
    for start, end in ((None, None), (S0, dS1)):
        got = lib.nugpr_decay_attention_backward(q, k, v, g, dev_off, do, scale=0.3, initial_state=start, d_final_state=end)
        want = reference_backward(q, k, v, g, off, 0.3, do, zero if start is None else start, zero if end is None else end)
        for x, w, name in zip(got, want, ("dq", "dk", "dv", "dS")):
            close(x, w, TOL[F32] if name == "dS" else TOL[dtype], name)


@pytest.mark.parametrize("layout", ["heads first", "odd"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides(lib, layout, dtype):
    lens = [70, 3, 130]
    q, k, v, do, g, off, dev_off, S0, dS1 = inputs(lens, 4, 2, 48, 40, dtype, seed=5, layout=layout)
    o, S = lib.nugpr_decay_attention_forward(q, k, v, g, dev_off, scale=1.0, initial_state=S0)
    want, end = reference(q, k, v, g, off, 1.0, S0)
    close(o, want, TOL[dtype])
    close(S, end, TOL[F32])
    got = lib.nugpr_decay_attention_backward(q, k, v, g, dev_off, do, initial_state=S0, d_final_state=dS1)
    for x, w, name in zip(got, reference_backward(q, k, v, g, off, 1.0, do, S0, dS1), ("dq", "dk", "dv", "dS")):
        close(x, w, TOL[F32] if name == "dS" else TOL[dtype], name)


def test_gradient_against_differences(lib):
    """Along one direction, central differences of the float64 reference: error h^2 of a cubic (q, k, v enter once each)."""
    lens = [5, 70, 0, 66]
    q, k, v, do, g, off, dev_off, S0, dS1 = inputs(lens, 4, 2, 24, 16, F32, seed=9)
    got = lib.nugpr_decay_attention_backward(q, k, v, g, dev_off, do, scale=0.5, initial_state=S0, d_final_state=dS1)
    gen = torch.Generator().manual_seed(1)
    base = [x.double().cpu() for x in (q, k, v, S0)]
    for which, name in enumerate(("q", "k", "v", "S0")):
        d = torch.randn(base[which].shape, generator=gen, dtype=torch.float64)
        f = []
        for sign in (1.0, -1.0):
            at = [x + sign * 1e-3 * d if j == which else x for j, x in enumerate(base)]
            o, S = reference(at[0], at[1], at[2], g, off, 0.5, at[3])
            f.append(float((o * do.double().cpu()).sum() + (S * dS1.double().cpu()).sum()))
        along = float((got[which].double().cpu() * d).sum())
        scale = float(got[which].double().norm()) * float(d.norm())
        assert abs(along - (f[0] - f[1]) / 2e-3) <= 64 * 2.0 ** -24 * scale, name


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_long_sequence(lib, dtype):
    """Many spans of one sequence beside short ones; the recurrence runs on the GPU, in float64."""
    lens = [4000, 1, 33000, 90]
    q, k, v, do, g, off, dev_off, S0, dS1 = inputs(lens, 2, 1, 128, 128, dtype, seed=2)
    g = torch.full((1,), -1.0 / 4096, device="cuda")
    o, S = lib.nugpr_decay_attention_forward(q, k, v, g, dev_off, scale=0.1, initial_state=S0)
    got = lib.nugpr_decay_attention_backward(q, k, v, g, dev_off, do, scale=0.1, initial_state=S0, d_final_state=dS1)
    # blocks of the definition: o = scale (decayed, masked Q K^T) V + decayed Q S0
    for s in range(len(lens)):
        a, b = int(off[s]), int(off[s + 1])
        Q, K, V, dO = (x[a:b].double() for x in (q, k, v, do))
        t = torch.arange(b - a, device="cuda", dtype=torch.float64)
        R = dS1[s, 0].double()
        dK, dV, dS = (torch.exp(g * (b - a - 1 - t))[:, None] * (V[:, 0] @ R.T), torch.exp(g * (b - a - 1 - t))[:, None] * (K[:, 0] @ R),
                      torch.exp(g * (b - a)) * R)
        want_o, want_dq = torch.zeros_like(dO), torch.zeros_like(Q)
        for h in range(2):
            w = torch.exp(g * (t + 1))[:, None]
            dS = dS + 0.1 * (w * Q[:, h]).T @ dO[:, h]
            for r0 in range(0, b - a, 4096):
                r = slice(r0, min(b - a, r0 + 4096))
                apart = t[r, None] - t[None, :]
                D = 0.1 * torch.exp(g * apart.clamp(min=0)) * (apart >= 0)
                P, dP = (Q[r, h] @ K[:, 0].T) * D, (dO[r, h] @ V[:, 0].T) * D
                want_o[r, h] = P @ V[:, 0] + 0.1 * w[r] * (Q[r, h] @ S0[s, 0].double())
                want_dq[r, h] = dP @ K[:, 0] + 0.1 * w[r] * (dO[r, h] @ S0[s, 0].double().T)
                dK += dP.T @ Q[r, h]
                dV += P.T @ dO[r, h]
        end = torch.exp(g * (b - a)) * S0[s, 0].double() + (torch.exp(g * (b - a - 1 - t))[:, None] * K[:, 0]).T @ V[:, 0]
        close(o[a:b], want_o.cpu(), TOL[dtype], "o")
        close(S[s, 0], end.cpu(), TOL[F32], "state")
        for x, w, name in ((got[0][a:b], want_dq, "dq"), (got[1][a:b, 0], dK, "dk"), (got[2][a:b, 0], dV, "dv")):
            close(x, w.cpu(), TOL[dtype], name)
        close(got[3][s, 0], dS.cpu(), TOL[F32], "dS")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_values_that_are_not_finite_stay_where_they_belong(lib, dtype):
    lens = [40, 200]
    q, k, v, do, g, off, dev_off, _, _ = inputs(lens, 2, 2, 64, 64, dtype, seed=4)
    want, _ = reference(q, k, v, g, off, 1.0)
    v2, k2, q2 = v.clone(), k.clone(), q.clone()
    v2[100, 0, 3] = float("nan")
    k2[120, 1, 5] = float("inf")
    q2[10, 0, 0] = float("nan")
    o, _ = lib.nugpr_decay_attention_forward(q2, k2, v2, g, dev_off)
    o = o.double().cpu()
    hit = torch.zeros(o.shape, dtype=torch.bool)
    hit[100:, 0, 3] = True                                     # every later token, this column
    hit[120:, 1, :] = True
    hit[10, 0, :] = True
    assert not torch.isfinite(o[hit]).any()
    close(o[~hit], want[~hit], TOL[dtype])
    # backwards: a gradient that is not finite reaches keys and values of earlier tokens only
    do2 = do.clone()
    do2[150, 1, 7] = float("nan")
    dq, dk, dv, _ = lib.nugpr_decay_attention_backward(q, k, v, g, dev_off, do2)
    zero = torch.zeros(2, 2, 64, 64)
    wq, wk, wv, _ = reference_backward(q, k, v, g, off, 1.0, do, zero, zero)
    assert torch.isfinite(dk[151:]).all() and torch.isfinite(dk[:40]).all() and torch.isfinite(dk[:, 0]).all()
    assert not torch.isfinite(dv[40:151, 1, 7]).any() and torch.isfinite(dv[151:]).all() and torch.isfinite(dv[:, 0]).all()
    close(dk[151:], wk[151:], TOL[dtype])
    close(dq[:150], wq[:150], TOL[dtype])


def test_decays_at_the_ends_of_their_range(lib):
    lens = [70, 65]
    q, k, v, do, _, off, dev_off, S0, dS1 = inputs(lens, 3, 3, 32, 32, F32, seed=6)
    g = torch.tensor([0.0, float("-inf"), -200.0], device="cuda")
    o, S = lib.nugpr_decay_attention_forward(q, k, v, g, dev_off, initial_state=S0)
    want, end = reference(q, k, v, g, off, 1.0, S0)
    close(o, want, TOL[F32])
    close(S, end, TOL[F32])
    got = lib.nugpr_decay_attention_backward(q, k, v, g, dev_off, do, initial_state=S0, d_final_state=dS1)
    for x, w in zip(got, reference_backward(q, k, v, g, off, 1.0, do, S0, dS1)):
        close(x, w, TOL[F32])


def test_rows_outside_the_sequences_are_zero_and_bad_offsets_harmless(lib):
    q, k, v, do, g, _, _, _, _ = inputs([200], 4, 2, 64, 64, F32, seed=7)
    off = np.array([20, 90, 150])
    dev = torch.from_numpy(off).cuda()
    filler = torch.full((200, 4, 64), float("nan"), device="cuda")
    del filler                                                   # (what the allocator hands out next)
    o, _ = lib.nugpr_decay_attention_forward(q, k, v, g, dev)
    want, _ = reference(q, k, v, g, off, 1.0)
    close(o, want, TOL[F32])
    got = lib.nugpr_decay_attention_backward(q, k, v, g, dev, do)
    for x in got[:3]:
        assert not x[:20].any() and not x[150:].any() and torch.isfinite(x).all()
    # beyond the ends: taken as the nearest end
    o2, S2 = lib.nugpr_decay_attention_forward(q, k, v, g, torch.tensor([-50, 90, 10 ** 15], device="cuda"))
    want, end = reference(q, k, v, g, [0, 90, 200], 1.0)
    close(o2, want, TOL[F32])
    close(S2, end, TOL[F32])


def test_states_may_share_memory_and_streams(lib):
    """Two halves through one state buffer equal the whole; on a stream of their own, with the inputs made there."""
    lens = [1000, 300]
    q, k, v, _, g, off, dev_off, S0, _ = inputs(lens, 2, 2, 64, 64, BF16, seed=8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        whole, end = lib.nugpr_decay_attention_forward(q, k, v, g, dev_off, initial_state=S0)
        S, parts = S0, []
        for a, b in ((0, 640), (640, 1000)):
            o, S = lib.nugpr_decay_attention_forward(q[a:b], k[a:b], v[a:b], g, torch.tensor([0, b - a, b - a], device="cuda"), initial_state=S)
            parts.append(o)
    torch.cuda.current_stream().wait_stream(side)
    close(torch.cat(parts), whole[:1000].double().cpu(), TOL[BF16])
    close(S[0], end[0].double().cpu(), TOL[F32])


def test_end_states_may_be_written_over_the_start_states(lib):
    """Through the C entry point: sequences of no span, of one and of many."""
    import ctypes as C

    from paper_2510_12128_amd import binding as B

    q, k, v, _, g, off, dev_off, S0, _ = inputs([0, 30, 3000], 4, 2, 48, 32, BF16, seed=13)
    want_o, want_S = lib.nugpr_decay_attention_forward(q, k, v, g, dev_off, initial_state=S0)
    c, o, S = B.load_library(), torch.empty_like(want_o), S0.clone()
    p = B.DecayAttention(B.NUGPR_BFLOAT16, 4, 2, 48, 32, q.shape[0], 3, dev_off.data_ptr(), g.data_ptr(), 1.0, None, 0)
    need = c.nugpr_decay_attention_workspace_bytes(C.byref(p), 0)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    p.workspace, p.workspace_bytes = ws.data_ptr(), need
    heads = [C.byref(B.Heads(x.data_ptr(), x.stride(0), x.stride(1))) for x in (q, k, v, o)]
    code = c.nugpr_decay_attention_forward(C.byref(p), *heads[:3], S.data_ptr(), heads[3], S.data_ptr(),
                                           torch.cuda.current_stream().cuda_stream)
    assert code == B.NUGPR_OK
    assert torch.equal(o, want_o) and torch.equal(S, want_S)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("h,kv,dk,dv", [(2, 2, 64, 64), (8, 2, 128, 128), (3, 3, 5, 17), (6, 1, 72, 36)])
def test_steps_continue_a_prompt(lib, h, kv, dk, dv, dtype):
    lens = [9, 40, 1]
    q, k, v, _, g, off, dev_off, S0, _ = inputs(lens, h, kv, dk, dv, dtype, seed=10)
    pool = torch.randn(6, kv, dk, dv, device="cuda")
    kept = pool.clone()
    slots = torch.tensor([4, 0, 3], dtype=torch.int32, device="cuda")
    pool[slots.long()] = S0
    o, S = reference(q, k, v, g, off, 0.7, S0)
    last = torch.from_numpy(off[1:] - 1).cuda()
    heads = [int(x) for x in off[1:] - 1]
    cut = np.concatenate([[0], np.cumsum(np.array(lens) - 1)]).astype(np.int64)
    rows = torch.tensor([t for s in range(3) for t in range(off[s], off[s + 1] - 1)], device="cuda")
    _, before = lib.nugpr_decay_attention_forward(q[rows], k[rows], v[rows], g, torch.from_numpy(cut).cuda(), scale=0.7, initial_state=S0)
    pool[slots.long()] = before
    got = lib.nugpr_decay_attention_step(q[last], k[last], v[last], g, pool, slots=slots, scale=0.7)
    close(got, o[heads], TOL[dtype])
    close(pool[slots.long()], S, TOL[F32])
    others = [1, 2, 5]
    assert torch.equal(pool[others], kept[others])


def test_step_passes_over_rows_without_a_request(lib):
    q, k, v, _, g, _, _, _, _ = inputs([4], 4, 2, 64, 64, F32, seed=11)
    pool = torch.randn(3, 2, 64, 64, device="cuda")
    kept = pool.clone()
    o = lib.nugpr_decay_attention_step(q, k, v, g, pool, slots=torch.tensor([-1, 2, 3, 2 ** 31 - 1], dtype=torch.int32, device="cuda"))
    assert not o[[0, 2, 3]].any() and o[1].any()
    assert torch.equal(pool[:2], kept[:2]) and not torch.equal(pool[2], kept[2])


def test_graph_replays(lib):
    q, k, v, do, g, off, dev_off, S0, dS1 = inputs([300, 50], 2, 2, 64, 64, BF16, seed=12)
    pool = S0.clone()
    lib.nugpr_decay_attention_forward(q, k, v, g, dev_off, initial_state=S0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, S = lib.nugpr_decay_attention_forward(q, k, v, g, dev_off, initial_state=S0)
        grads = lib.nugpr_decay_attention_backward(q, k, v, g, dev_off, do, initial_state=S0, d_final_state=dS1)
        one = lib.nugpr_decay_attention_step(q[:2], k[:2], v[:2], g, pool)
    for r in range(3):
        q.copy_(torch.randn(q.shape, device="cuda"))
        before = pool.clone()
        graph.replay()
        torch.cuda.synchronize()
        again = lib.nugpr_decay_attention_forward(q, k, v, g, dev_off, initial_state=S0)
        assert torch.equal(o, again[0]) and torch.equal(S, again[1])
        for x, y in zip(grads, lib.nugpr_decay_attention_backward(q, k, v, g, dev_off, do, initial_state=S0, d_final_state=dS1)):
            assert torch.equal(x, y)
        assert torch.equal(one, lib.nugpr_decay_attention_step(q[:2], k[:2], v[:2], g, before)) and torch.equal(before, pool)


def test_no_rows_and_no_sequences(lib):
    q, k, v, do, g, _, _, S0, dS1 = inputs([3], 2, 2, 16, 16, F32)
    none = torch.zeros(1, dtype=torch.int64, device="cuda")
    o, S = lib.nugpr_decay_attention_forward(q[:0], k[:0], v[:0], g, none)
    assert o.shape == (0, 2, 16) and S.shape == (0, 2, 16, 16)
    empty = torch.zeros(2, dtype=torch.int64, device="cuda")
    o, S = lib.nugpr_decay_attention_forward(q[:0], k[:0], v[:0], g, empty, initial_state=S0)
    assert torch.equal(S, S0)
    got = lib.nugpr_decay_attention_backward(q[:0], k[:0], v[:0], g, empty, do[:0], initial_state=S0, d_final_state=dS1)
    assert torch.equal(got[3], dS1)
    assert lib.nugpr_decay_attention_step(q[:0], k[:0], v[:0], g, S0).shape == (0, 2, 16)


def test_refusals(lib):
    q, k, v, do, g, off, dev_off, S0, _ = inputs([8], 4, 2, 16, 16, F32)
    fwd, step = lib.nugpr_decay_attention_forward, lib.nugpr_decay_attention_step
    bad = [
        lambda: fwd(q.half(), k.half(), v.half(), g, dev_off),
        lambda: fwd(q, k.to(BF16), v, g, dev_off),
        lambda: fwd(q[:, :3], k, v, g, dev_off),                    # 3 heads over 2
        lambda: fwd(q, k, v[:7], g, dev_off),
        lambda: fwd(q, k, v, g[:1], dev_off),
        lambda: fwd(q, k, v, g.double(), dev_off),
        lambda: fwd(q, k, v, g, dev_off.int()),
        lambda: fwd(q, k, v, g, dev_off.cpu()),
        lambda: fwd(q, k, v, g, dev_off, scale=float("nan")),
        lambda: fwd(q, k, v, g, dev_off, initial_state=S0[:, :1]),
        lambda: fwd(q, k, v, g, dev_off, initial_state=S0.to(BF16)),
        lambda: fwd(q.transpose(1, 2), k.transpose(1, 2), v, g, dev_off),
        lambda: fwd(torch.zeros(8, 2, 129, device="cuda"), torch.zeros(8, 2, 129, device="cuda"), v, g, dev_off),
        lambda: lib.nugpr_decay_attention_backward(q, k, v, g, dev_off, do[:, :2]),
        lambda: step(q, k, v, g, S0),                               # eight requests, one state
        lambda: step(q, k, v, g, S0.transpose(2, 3), slots=torch.zeros(8, dtype=torch.int32, device="cuda")),
        lambda: step(q, k, v, g, S0, slots=torch.zeros(8, dtype=torch.int64, device="cuda")),
    ]
    for f in bad:
        with pytest.raises(lib.NugprError):
            f()
