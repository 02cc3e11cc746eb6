"""An infinite value, or a NaN, among the inputs of the sequence operators (GPU) makes the results that the formulas give it, infinities and NaN alike,
by the definitions in float64; what it does not reach stays as it is.  Inputs are positive, so that infinities of one sign do not
cancel by the order of a sum.

Tolerances of the finite rest, relative in the 2-norm: sums of up to 5400 positive terms, each rounded by 2^-24 at most, all in one
direction at worst: 2^-11; bfloat16 outputs 2^-8 more, within 2^-7."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
TOL = {F32: 2.0 ** -11, BF16: 2.0 ** -7}
INF = float("inf")


def alike(x, want, tol, name):
    x, want = x.double().cpu(), want.double().cpu()
    assert torch.equal(torch.isnan(x), torch.isnan(want)), (name, "NaN", int(torch.isnan(x).sum()), int(torch.isnan(want).sum()))
    for sign in (INF, -INF):
        assert torch.equal(x == sign, want == sign), (name, sign, int((x == sign).sum()), int((want == sign).sum()))
    fine = torch.isfinite(want)
    assert float((x[fine] - want[fine]).norm()) <= tol * float(want[fine].norm()), name


def recurrence(q, k, v, g, offsets, S0):
    q, k, v, g, S0 = (x.double().cuda() for x in (q, k, v, g, S0))
    lam, kv, dk, dv = torch.exp(g)[:, None, None], k.shape[1], k.shape[2], v.shape[2]
    o, ends = torch.zeros(q.shape[0], q.shape[1], dv, dtype=torch.float64, device="cuda"), S0.clone()
    for s in range(len(offsets) - 1):
        for t in range(offsets[s], offsets[s + 1]):
            ends[s] = lam * ends[s] + k[t][:, :, None] * v[t][:, None, :]
            o[t] = (q[t].reshape(kv, -1, dk, 1) * ends[s][:, None]).sum(2).reshape(-1, dv)      # (a product would add zeros' multiples)
    return o, ends


def recurrence_backward(q, k, v, g, offsets, do, S0, R):
    q, k, v, g, do, S0, R = (x.double().cuda() for x in (q, k, v, g, do, S0, R))
    lam, kv, dk, dv = torch.exp(g)[:, None, None], k.shape[1], k.shape[2], v.shape[2]
    dq, dk_, dv_, U = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v), R.clone()
    S = S0.clone()
    for s in range(len(offsets) - 1):
        for t in range(offsets[s], offsets[s + 1]):
            S[s] = lam * S[s] + k[t][:, :, None] * v[t][:, None, :]
            dq[t] = (do[t].reshape(kv, -1, 1, dv) * S[s][:, None]).sum(3).reshape(-1, dk)
        for t in reversed(range(offsets[s], offsets[s + 1])):
            U[s] = U[s] + (q[t].reshape(kv, -1, dk, 1) * do[t].reshape(kv, -1, 1, dv)).sum(1)
            dk_[t] = (U[s] * v[t][:, None, :]).sum(2)
            dv_[t] = (U[s] * k[t][:, :, None]).sum(1)
            U[s] = lam * U[s]
    return dq, dk_, dv_, U


def positive(gen, *shape):
    return torch.rand(*shape, generator=gen) + 0.5


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [INF, float("nan")])
@pytest.mark.parametrize("where", ["k", "v", "q", "initial_state"])
@pytest.mark.parametrize("h,kv,dk,dv", [(2, 2, 64, 64), (6, 3, 40, 72), (4, 2, 128, 128), (3, 3, 5, 17), (96, 96, 20, 24)])      # (many heads: spans of several blocks)
def test_attention(lib, h, kv, dk, dv, where, bad, dtype):
    lens = [40, 0, 2300, 1, 90]                       # one block, none, many spans, one token, two blocks
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    gen = torch.Generator().manual_seed(dk)
    n = int(off[-1])
    q, k, v = (positive(gen, n, x, w).to(dtype) for x, w in ((h, dk), (kv, dk), (kv, dv)))
    S0 = positive(gen, len(lens), kv, dk, dv)
    for t in (10, 50, 1500, int(off[4]) + 70):
        if where == "k":
            k[t, ::2, t % dk] = bad
        elif where == "v":
            v[t, ::2, t % dv] = bad
            v[t + 3, 1::2, (t + 1) % dv] = -bad
        elif where == "q":
            q[t, h - 1, t % dk] = bad
    if where == "initial_state":
        S0[0, 0, 1, 2], S0[2, kv - 1, 3, 1], S0[3, 0, 2, 2] = bad, -bad, bad
    g = torch.log1p(-2.0 ** -torch.linspace(7, 10, kv))
    args = [x.cuda() for x in (q, k, v, g, torch.from_numpy(off))]
    o, S = lib.nugpr_decay_attention_forward(*args, initial_state=S0.cuda())
    want_o, want_S = recurrence(q, k, v, g, off, S0)
    alike(S, want_S, TOL[F32], "state")
    alike(o, want_o, TOL[dtype], "o")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [INF, float("nan")])
@pytest.mark.parametrize("where", ["k", "v", "do"])
@pytest.mark.parametrize("h,kv,dk,dv", [(2, 2, 64, 64), (6, 3, 40, 72), (4, 2, 128, 128)])
def test_attention_gradients(lib, h, kv, dk, dv, where, bad, dtype):
    lens = [40, 0, 500, 1, 90]
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    gen = torch.Generator().manual_seed(dk + 1)
    n = int(off[-1])
    q, k, v, do = (positive(gen, n, x, w).to(dtype) for x, w in ((h, dk), (kv, dk), (kv, dv), (h, dv)))
    S0, R = positive(gen, len(lens), kv, dk, dv), positive(gen, len(lens), kv, dk, dv)
    for t in (10, 250, int(off[4]) + 70):
        {"k": k, "v": v, "do": do}[where][t, 0, t % min(dk, dv)] = bad
    g = torch.log1p(-2.0 ** -torch.linspace(7, 10, kv))
    args = [x.cuda() for x in (q, k, v, g, torch.from_numpy(off), do)]
    got = lib.nugpr_decay_attention_backward(*args, initial_state=S0.cuda(), d_final_state=R.cuda())
    want = recurrence_backward(q, k, v, g, off, do, S0, R)
    for x, w, name in zip(got, want, ("dq", "dk", "dv", "d_initial_state")):
        alike(x, w, TOL[F32] if name == "d_initial_state" else TOL[dtype], name)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dk,dv", [(64, 64), (40, 128)])
def test_what_leaves_the_range_of_float32_is_infinite(lib, dk, dv, dtype):
    """Finite keys and values whose product is not, and a finite query whose product with the state is not."""
    lens = [50, 400, 3]
    gen, off = torch.Generator().manual_seed(5), np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    q, k, v = (positive(gen, 453, 2, w).to(dtype) for w in (dk, dk, dv))
    k[60, 0], v[60, 0, 3:] = 1e25, 1e25
    q[200, 1], q[449, 1] = 1e38, 1e38
    g, S0 = torch.tensor([-0.001, -0.002]), positive(gen, 3, 2, dk, dv)
    o, S = lib.nugpr_decay_attention_forward(q.cuda(), k.cuda(), v.cuda(), g.cuda(), torch.from_numpy(off).cuda(), initial_state=S0.cuda())
    want_o, want_S = recurrence(q, k, v, g, off, S0)
    want_o, want_S = want_o.cpu(), want_S.cpu()                            # (1e50 and 1e42 in float64)
    want_o[want_o > 3.5e38], want_S[want_S > 3.5e38] = INF, INF
    assert int(want_S.isinf().sum()) == dk * (dv - 3) and int(want_o.isinf().sum()) == 390 * (dv - 3) + 2 * dv
    # (row 60 of the first three columns has a key of 1e25: of another size than all other results, so it is compared alone)
    far = want_o > 1e20
    far &= want_o.isfinite()
    alike(torch.where(far, torch.zeros(()), o.cpu().double()), torch.where(far, torch.zeros(()), want_o), TOL[dtype], "o")
    assert torch.allclose(o.cpu().double()[far], want_o[far], rtol=TOL[dtype], atol=0)
    small = want_S < 1e20
    alike(torch.where(small, S.cpu().double(), torch.zeros(())), torch.where(small, want_S, torch.zeros(())), TOL[F32], "state")
    assert torch.equal(S.cpu().isinf(), want_S.isinf())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_step_keeps_an_infinite_state(lib, dtype):
    gen = torch.Generator().manual_seed(3)
    q, k, v = (positive(gen, 3, 2, 16).to(dtype) for _ in range(3))
    S0 = positive(gen, 3, 2, 16, 16)
    S0[0, 0, 1, 2], S0[1, 1, 3, 3] = INF, -INF
    v[2, 0, 5] = INF
    g = torch.tensor([0.0, -0.3])
    S = S0.cuda()
    o = lib.nugpr_decay_attention_step(q.cuda(), k.cuda(), v.cuda(), g.cuda(), S)
    want_o, want_S = recurrence(q, k, v, g, [0, 1, 2, 3], S0)
    alike(S, want_S, TOL[F32], "state")
    alike(o, want_o, TOL[dtype], "o")


def adapted(x, W, A, B, off, which, dy):
    x, W, A, B, dy = (t.double().cpu() for t in (x, W, A, B, dy))
    y, dx, dA, dB = x @ W.T, dy @ W, torch.zeros_like(A), torch.zeros_like(B)
    for s, a in enumerate(which):
        r = slice(int(off[s]), int(off[s + 1]))
        low, up = x[r] @ A[a].T, dy[r] @ B[a].T
        y[r] += low @ B[a]
        dx[r] += up @ A[a]
        dA[a] += up.T @ x[r]
        dB[a] += low.T @ dy[r]
    return y, dx, dA, dB


@pytest.mark.parametrize("whole", [False, True], ids=["spread", "ones"])     # (ones: low parts of h are zero)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("where", ["x", "dy", "A", "B", "W"])
@pytest.mark.parametrize("lens,inp,out,rank", [
    ([5, 9, 30], 64, 80, 4), ([5, 9, 400], 64, 80, 33), ([5, 90, 400], 256, 40, 8), ([4] * 70, 130, 203, 20), ([700, 20, 800], 256, 1088, 3),
    ([1, 300, 5400], 192, 2104, 2), ([1, 300, 2600], 192, 2104, 40)], ids=lambda x: str(sum(x)) if isinstance(x, list) else str(x))
def test_adapters(lib, lens, inp, out, rank, where, dtype, whole):
    gen = torch.Generator().manual_seed(inp + rank)
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    n, which = int(off[-1]), [s % 3 for s in range(len(lens))]

    def some(*shape):
        return (torch.ones(*shape) if whole else positive(gen, *shape)).to(dtype)

    x, W, A, B, dy = some(n, inp), some(out, inp), some(3, rank, inp), some(3, rank, out), some(n, out)
    if where == "x":
        x[2, 7], x[n - 3, 0] = INF, -INF
    elif where == "dy":
        dy[2, 7], dy[n - 3, 0] = INF, -INF
    elif where == "A":
        A[1, rank - 1, 5] = INF
    elif where == "B":
        B[1, 0, 5] = -INF
    else:
        W[3, 4] = INF
    args = [t.cuda() for t in (x, W, A, B, torch.from_numpy(off))]
    dev_which = torch.tensor(which, dtype=torch.int32, device="cuda")
    got = (lib.nugpr_adapter_forward(*args, adapter_of=dev_which), *lib.nugpr_adapter_backward(*args, dy.cuda(), adapter_of=dev_which))
    for g, w, name in zip(got, adapted(x, W, A, B, off, which, dy), ("y", "dx", "dA", "dB")):
        alike(g, w, TOL[dtype], name)
