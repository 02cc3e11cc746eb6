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
