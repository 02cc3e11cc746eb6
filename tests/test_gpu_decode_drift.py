"""Thousands of single tokens on one slowly decaying state (GPU), against the recurrence in float64 and the same tokens as a prompt.

Tolerance, relative in the 2-norm: the recurrence in float32 rounds a state once a token, 2^-24 at most, independent from token to token, and a
state remembers up to 10^4 tokens: 64 x 2^-24 as for the prompt (100 of them, each half as large on average and less for the newer ones)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TOL = 64 * 2.0 ** -24


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_steps_do_not_drift_from_the_prompt(lib, dtype):
    n, kv, dk, dv = 6000, 4, 16, 12
    gen = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(n, kv, w, generator=gen).to(dtype).cuda() for w in (dk, dk, dv))
    S0 = torch.randn(1, kv, dk, dv, generator=gen).cuda()
    g = torch.log(torch.tensor([0.999, 0.9995, 0.9999, 1 - 2.0 ** -12], dtype=torch.float64)).float().cuda()
    state, exact, lam = S0.clone(), S0[0].double(), torch.exp(g.double())[:, None, None]
    k64, v64 = k.double(), v.double()
    for t in range(n):
        lib.nugpr_decay_attention_step(q[t:t + 1], k[t:t + 1], v[t:t + 1], g, state)
        exact = lam * exact + k64[t][:, :, None] * v64[t][:, None, :]
    _, prompt = lib.nugpr_decay_attention_forward(q, k, v, g, torch.tensor([0, n], device="cuda"), initial_state=S0)
    for j in range(kv):
        for got, name in ((prompt[0, j], "prompt"), (state[0, j], "steps")):
            err = float((got.double() - exact[j]).norm() / exact[j].norm())
            assert err <= TOL, (name, float(g[j]), err)
