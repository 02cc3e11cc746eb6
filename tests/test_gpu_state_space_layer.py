"""The convolution, the scan and the clipping together (GPU), as a layer that is trained and then answers token by token:
examples/state_space_regression.py.

The example is tested for running, for its layer's gradients, and for single tokens that give what whole sequences give; not
for how far its loss falls."""
import importlib.util
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("state_space_regression", os.path.join(ROOT, "examples", "state_space_regression.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_the_example_runs(lib, example):
    out = example.main(steps=20)
    assert np.isfinite(out["losses"]).all() and np.isfinite(out["norms"]).all() and np.isfinite(out["nll"]).all()
    assert np.isfinite(out["rmse"]).all()
    # windows are the same numbers; a state one rounding a token off, and sums of 24 and 6 products in torch's own order for another
    # number of rows: roundings of 2^-24 each, some 200 of them at most, in one direction at worst
    assert out["apart"] < 256 * 2.0 ** -24


def plain(layer, m, tokens, offsets):
    """The layer's coordinates from its formulas, in the type of its parameters."""
    p = tokens @ layer["W"]
    x, z, dt, B, C = p.split([m.DIM, m.DIM, m.DIM, m.STATES, m.STATES], dim=1)
    A, out = -torch.exp(layer["log_A"]), []
    for lo, hi in zip(offsets[:-1], offsets[1:]):
        h, y = torch.zeros(m.DIM, m.STATES, dtype=x.dtype), None
        for t in range(lo, hi):
            q = layer["bias"] + sum(layer["taps"][:, m.TAPS - 1 - k] * x[t - k] for k in range(m.TAPS) if t - k >= lo)
            u = q * torch.sigmoid(q)
            d = torch.log1p(torch.exp(dt[t] + layer["dt_bias"]))
            h = torch.exp(d[:, None] * A) * h + (d * u)[:, None] * B[t]
            y = ((C[t] * h).sum(1) + layer["D"] * u) * z[t] * torch.sigmoid(z[t])
        out.append(y @ layer["R"])
    return torch.stack(out)


def test_gradients_through_the_layer(lib, example):
    """Against autograd of the formulas in 64 bits.  Every parameter's gradient passes through sums of some hundred products in
    each of four operators, each rounding 2^-24 and independent of the others: below 2^-15 of the whole, relative in the 2-norm."""
    m = example
    layer = m.Layer(3, "cuda:0")
    gen = torch.Generator().manual_seed(4)
    lens = [5, 90, 1, 33]
    off = np.concatenate([[0], np.cumsum(lens)])
    tokens, y = torch.randn(sum(lens), m.WIDTH, generator=gen), torch.randn(len(lens), generator=gen)
    coords, _, _ = layer.forward(tokens.cuda(), torch.from_numpy(off).cuda())
    (coords @ layer.r - y.cuda()).square().mean().backward()
    names = ["W", "taps", "bias", "dt_bias", "log_A", "D", "R", "r"]
    exact = {k: getattr(layer, k).detach().double().cpu().requires_grad_() for k in names}
    want = plain(exact, m, tokens.double(), off)
    (want @ exact["r"] - y.double()).square().mean().backward()
    assert float((coords.detach().double().cpu() - want.detach()).norm()) <= 2.0 ** -15 * float(want.detach().norm())
    for k, p in zip(names, layer.trained()):
        got, w = p.grad.double().cpu(), exact[k].grad
        assert float((got - w).norm()) <= 2.0 ** -15 * float(w.norm()), k
    # clipped together: one norm over all of them
    grads = [p.grad.clone() for p in layer.trained()]
    norm = float(sum(exact[k].grad.square().sum() for k in names).sqrt())
    got = lib.nugpr_clip_gradients([p.grad for p in layer.trained()], 0.5 * norm)
    assert abs(float(got) - norm) <= 2.0 ** -15 * norm
    for p, g in zip(layer.trained(), grads):
        assert float((p.grad - 0.5 * g).norm()) <= 2.0 ** -14 * float(g.norm())


def test_a_sequence_in_two_calls(lib, example):
    """The second call goes on from the first one's windows and states, and its gradient comes back through them."""
    m = example
    layer = m.Layer(5, "cuda:0")
    tokens = torch.randn(150, m.WIDTH, generator=torch.Generator().manual_seed(6)).cuda()

    def offsets(*o):
        return torch.tensor(o, device="cuda")

    def gradients(coords):
        grads = torch.autograd.grad(coords.square().sum(), layer.trained()[:-1])
        return coords.detach(), grads

    whole, want = gradients(layer.forward(tokens, offsets(0, 100, 150))[0])
    # (both sequences' first halves, then the rest)
    first = torch.cat([tokens[:37], tokens[100:120]])
    rest = torch.cat([tokens[37:100], tokens[120:]])
    _, window, state = layer.forward(first, offsets(0, 37, 57))
    parts, got = gradients(layer.forward(rest, offsets(0, 63, 93), window, state)[0])
    assert float((parts - whole).norm()) <= 2.0 ** -16 * float(whole.norm())
    for g, w in zip(got, want):
        assert float((g - w).norm()) <= 2.0 ** -15 * float(w.norm())
