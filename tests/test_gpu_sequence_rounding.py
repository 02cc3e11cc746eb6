"""What the bfloat16 sequence operators (GPU) round: their outputs, once, and nothing before.

Every result is compared with float64 on the same inputs.  `once` is the error of that result itself, rounded to bfloat16: what
no kernel can beat.  A kernel may add to it what float32 sums leave behind, in the 2-norm: 1 / 50 of it where nothing cancels,
8 x 2^-24 of the terms where they do (sums of at most 256 products, whose 2^-24 each grow with the square root at
most, halved as rounding errors are spread evenly)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def once(want):
    return float((want.to(BF16).double() - want).norm())


def decayed(q, k, v, g, S0):
    """o and end state of one sequence and head, scale 1, in float64."""
    t = torch.arange(q.shape[0], device=q.device, dtype=torch.float64)
    apart = t[:, None] - t[None, :]
    D = torch.exp(g * apart.clamp(min=0)) * (apart >= 0)
    return ((q @ k.T) * D) @ v + torch.exp(g * (t + 1))[:, None] * (q @ S0), D


@pytest.mark.parametrize("n", [1, 50, 64, 700])
@pytest.mark.parametrize("h,kv,dk,dv", [(2, 2, 64, 64), (4, 1, 128, 128), (3, 3, 40, 17), (4, 2, 128, 72)])
def test_attention_rounds_its_outputs_alone(lib, n, h, kv, dk, dv):
    gen = torch.Generator().manual_seed(n + dk)

    def r(*shape):
        return torch.randn(*shape, generator=gen).cuda()

    q, k, v, do = (x.to(BF16) for x in (r(n, h, dk), r(n, kv, dk), r(n, kv, dv), r(n, h, dv)))
    S0, R = r(1, kv, dk, dv), r(1, kv, dk, dv)
    g = torch.log1p(-2.0 ** -torch.linspace(3, 10, kv)).cuda()
    off = torch.tensor([0, n], device="cuda")
    o, _ = lib.nugpr_decay_attention_forward(q, k, v, g, off, initial_state=S0)
    dq, dk_, dv_, _ = lib.nugpr_decay_attention_backward(q, k, v, g, off, do, initial_state=S0, d_final_state=R)
    t = torch.arange(n, device="cuda", dtype=torch.float64)
    want_o, want_dq = torch.zeros(n, h, dv, dtype=torch.float64, device="cuda"), torch.zeros(n, h, dk, dtype=torch.float64, device="cuda")
    want_dk, want_dv = torch.zeros(n, kv, dk, dtype=torch.float64, device="cuda"), torch.zeros(n, kv, dv, dtype=torch.float64, device="cuda")
    for j in range(kv):
        lam, K, V, S, U = g[j].double(), k[:, j].double(), v[:, j].double(), S0[0, j].double(), R[0, j].double()
        w = torch.exp(lam * (n - 1 - t))[:, None]
        want_dk[:, j] = w * (V @ U.T)
        want_dv[:, j] = w * (K @ U)
        for x in range(j * (h // kv), (j + 1) * (h // kv)):
            Q, dO = q[:, x].double(), do[:, x].double()
            want_o[:, x], D = decayed(Q, K, V, lam, S)
            want_dq[:, x], _ = decayed(dO, V, K, lam, S.T)
            want_dk[:, j] += ((dO @ V.T) * D).T @ Q
            want_dv[:, j] += ((Q @ K.T) * D).T @ dO
    for got, want, name in ((o, want_o, "o"), (dq, want_dq, "dq"), (dk_, want_dk, "dk"), (dv_, want_dv, "dv")):
        assert float((got.double() - want).norm()) <= 1.02 * once(want), name


# (rows, width in, width out, rank): few rows; small tiles; larger ones; tiles of 128 and of 256 rows in bfloat16; few columns
SHAPES = [(40, 96, 64, 2), (300, 256, 264, 3), (301, 253, 259, 20), (1500, 256, 1088, 2), (2900, 192, 2104, 2), (5700, 192, 2104, 33),
          (5700, 200, 1000, 2), (400, 256, 24, 2)]


def nearly_twice(gen, n, width):
    """Rows in pairs, the second with one value moved by a rounding step of bfloat16."""
    a = torch.randn(n, width, generator=gen).to(BF16)
    b = a.clone()
    at = torch.randint(0, width, (n, 1), generator=gen)
    b.scatter_(1, at, (a.gather(1, at).float() * (1 + 2.0 ** -7)).to(BF16))
    return a, b


def held(got, want, terms):
    err = float((got.double().cpu() - want).norm())
    assert err <= 1.02 * once(want) + 8 * 2.0 ** -24 * float(terms.norm()), (err / float(want.norm()), once(want) / float(want.norm()))


@pytest.mark.parametrize("requests", [1, 40])
@pytest.mark.parametrize("n,inp,out,rank", SHAPES)
def test_low_rank_rows_keep_float32(lib, n, inp, out, rank, requests):
    """y = (h_0 - h_1) b with h_1 within 2^-12 of h_0, and dx alike: what h loses shows 2^12 times."""
    gen = torch.Generator().manual_seed(n + rank)
    x, dy = torch.randn(n, inp, generator=gen).to(BF16), torch.randn(n, out, generator=gen).to(BF16)
    off = torch.from_numpy(np.linspace(0, n, requests + 1).astype(np.int64)).cuda()
    which = torch.zeros(requests, dtype=torch.int32, device="cuda")
    W = torch.zeros(out, inp, dtype=BF16)

    def adapter(width, same):
        a = torch.zeros(1, rank, width, dtype=BF16)
        if same:
            a[0, 0] = torch.randn(width, generator=gen).to(BF16)
            a[0, 1] = -a[0, 0]
        else:
            first, second = nearly_twice(gen, 1, width)
            a[0, 0], a[0, 1] = first[0], second[0]
        return a

    A, B = adapter(inp, False), adapter(out, True)
    y = lib.nugpr_adapter_forward(x.cuda(), W.cuda(), A.cuda(), B.cuda(), off, adapter_of=which)
    low = x.double() @ A[0, :2].double().T
    held(y, low @ B[0, :2].double(), low[:, :1] @ B[0, :1].double())
    A, B = adapter(inp, True), adapter(out, False)
    dx = lib.nugpr_adapter_backward(x.cuda(), W.cuda(), A.cuda(), B.cuda(), off, dy.cuda(), adapter_of=which)[0]
    up = dy.double() @ B[0, :2].double().T
    held(dx, up @ A[0, :2].double(), up[:, :1] @ A[0, :1].double())


@pytest.mark.parametrize("pairs,inp,out,rank", [(32, 256, 256, 1), (500, 253, 130, 20), (700, 256, 136, 40), (90, 250, 256, 100)])
def test_sums_over_rows_keep_float32(lib, pairs, inp, out, rank):
    """dB = sum (h_t - h_t') dy_t over pairs of rows, and dA alike."""
    gen = torch.Generator().manual_seed(pairs + rank)
    off = torch.tensor([0, 2 * pairs], device="cuda")
    W, A, B = (torch.randn(*s, generator=gen).to(BF16) for s in ((out, inp), (1, rank, inp), (1, rank, out)))
    for of_A in (False, True):
        first, second = nearly_twice(gen, pairs, out if of_A else inp)
        other = torch.randn(pairs, inp if of_A else out, generator=gen).to(BF16)
        order = torch.arange(2 * pairs).reshape(2, pairs).T.reshape(-1)           # the two rows of a pair side by side
        near, signed = torch.cat([first, second])[order], torch.cat([other, -other])[order]
        x, dy = (signed, near) if of_A else (near, signed)
        _, dA, dB = lib.nugpr_adapter_backward(x.cuda(), W.cuda(), A.cuda(), B.cuda(), off, dy.cuda())
        low = near.double() @ (B if of_A else A)[0].double().T
        want = low.T @ signed.double()
        terms = float((low ** 2).sum(0).sqrt().norm()) * float(signed.double().norm()) / (2 * pairs) ** 0.5
        held((dA if of_A else dB)[0], want, torch.tensor(terms))
