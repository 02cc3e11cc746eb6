"""Regression on sequences: a state space layer makes the coordinates, the Gaussian process regresses on them; later tokens
arrive one at a time.

  1. The layer (a projection, the short causal convolution, the selective scan, a linear readout of a sequence's last token) is
     fitted by gradient descent, its gradients clipped to a common norm (nugpr_short_conv_*, nugpr_selective_scan_*,
     nugpr_clip_gradients).  Each operator is an autograd function here, its gradient the operator's own _backward call.
  2. The readout's coordinates of every sequence go into a Context: training steps, predictions for held-out sequences.
  3. Held-out sequences grow by a token each: a step of the convolution and of the scan on the kept windows and states, a new
     prediction.  The same coordinates come out as from the whole sequences.

Run: python examples/state_space_regression.py"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2510_12128_amd as P  # noqa: E402

CLUSTERS, PER, WIDTH, DIM, STATES, TAPS, COORDS = 4, 256, 6, 24, 8, 3, 3


class ShortConv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, offsets, window):
        ctx.save_for_backward(x, weight, bias, offsets, window)
        return P.nugpr_short_conv_forward(x, weight, offsets, bias=bias, silu=True, initial_state=window)

    @staticmethod
    def backward(ctx, d_y, d_end):
        x, weight, bias, offsets, window = ctx.saved_tensors
        dx, dw, db, ds = P.nugpr_short_conv_backward(x, weight, offsets, d_y.contiguous(), bias=bias, silu=True,
                                                     initial_state=window, d_final_state=d_end.contiguous())
        return dx, dw, db, None, None if window is None else ds


class SelectiveScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, dt, A, B, C, D, z, dt_bias, offsets, state):
        ctx.save_for_backward(x, dt, A, B, C, D, z, dt_bias, offsets, state)
        return P.nugpr_selective_scan_forward(x, dt, A, B, C, offsets, D=D, z=z, dt_bias=dt_bias, initial_state=state)

    @staticmethod
    def backward(ctx, d_y, d_end):
        x, dt, A, B, C, D, z, dt_bias, offsets, state = ctx.saved_tensors
        *d, ds = P.nugpr_selective_scan_backward(x, dt, A, B, C, offsets, d_y.contiguous(), D=D, z=z, dt_bias=dt_bias,
                                                 initial_state=state, d_final_state=d_end.contiguous())
        return *d, None, None if state is None else ds


class Layer:
    """token -> [x | z | dt | B | C] by a projection; x through the convolution and the scan, gated by z; the last token's readout."""

    def __init__(self, seed, device, dtype=torch.float32):
        g = torch.Generator(device=device).manual_seed(seed)

        def r(*shape, scale):
            return (torch.randn(*shape, generator=g, device=device) * scale).to(dtype)

        self.W = r(WIDTH, 3 * DIM + 2 * STATES, scale=WIDTH ** -0.5)
        self.taps, self.bias = r(DIM, TAPS, scale=TAPS ** -0.5), r(DIM, scale=0.1)
        steps = torch.exp(torch.rand(DIM, generator=g, device=device) * 3.0 - 4.0)             # 0.02 to 0.4
        self.dt_bias = torch.log(torch.expm1(steps))
        self.log_A = torch.log(torch.arange(1, STATES + 1, device=device, dtype=torch.float32)).repeat(DIM, 1)
        self.D = torch.ones(DIM, device=device)
        self.R = r(DIM, COORDS, scale=DIM ** -0.5)
        self.r = r(COORDS, scale=1.0)
        for p in self.trained():
            p.requires_grad_()

    def trained(self):
        return [self.W, self.taps, self.bias, self.dt_bias, self.log_A, self.D, self.R, self.r]

    def split(self, tokens):
        p = tokens @ self.W
        x, z, dt, B, C = p.split([DIM, DIM, DIM, STATES, STATES], dim=1)                       # (views)
        return x, z, dt, B.unsqueeze(1), C.unsqueeze(1)

    def forward(self, tokens, offsets, window=None, state=None):
        """Coordinates of the sequences, and their windows and states at the end."""
        x, z, dt, B, C = self.split(tokens)
        x, window = ShortConv.apply(x, self.taps, self.bias, offsets, window)
        y, state = SelectiveScan.apply(x, dt, -torch.exp(self.log_A), B, C, self.D, z, self.dt_bias, offsets, state)
        return y[offsets[1:] - 1] @ self.R, window, state

    @torch.no_grad()
    def step(self, tokens, window, state):
        """One more token of each sequence; windows and states go on in place."""
        x, z, dt, B, C = self.split(tokens)
        x = P.nugpr_short_conv_step(x, self.taps, window, bias=self.bias, silu=True)
        y = P.nugpr_selective_scan_step(x, dt, -torch.exp(self.log_A), B, C, state, D=self.D, z=z, dt_bias=self.dt_bias)
        return y @ self.R


def data(seed, per, device):
    """Sequences cluster by cluster; the target of one is what its tokens leave in a sum that forgets faster after tokens whose
    second entry is large."""
    rng = np.random.default_rng(seed)
    along = np.random.default_rng(11).normal(size=(CLUSTERS, WIDTH)) / WIDTH ** 0.5
    tokens, targets = [], []
    for c in range(CLUSTERS):
        for _ in range(per):
            x = rng.normal(size=(int(rng.integers(4, 40)), WIDTH))
            x[:, 0] = 1.0
            h = np.zeros(WIDTH)
            for t in x:
                h = np.exp(-0.3 / (1.0 + np.exp(-2.0 * t[1]))) * h + t
            targets.append(h @ along[c] * 0.5 + rng.normal() * 0.02)
            tokens.append(x)
    offsets = np.concatenate([[0], np.cumsum([len(x) for x in tokens])]).astype(np.int64)
    return (torch.tensor(np.concatenate(tokens), dtype=torch.float32, device=device), torch.from_numpy(offsets).to(device),
            torch.arange(CLUSTERS, device=device).repeat_interleave(per),
            torch.tensor(np.array(targets), dtype=torch.float32, device=device))


def fit(layer, tokens, offsets, y, steps, bound=1.0):
    optimiser = torch.optim.Adam(layer.trained(), lr=0.01)
    losses, norms = [], []
    for _ in range(steps):
        optimiser.zero_grad()
        coords, _, _ = layer.forward(tokens, offsets)
        loss = (coords @ layer.r - y).square().mean()
        loss.backward()
        norms.append(P.nugpr_clip_gradients([p.grad for p in layer.trained()], bound))
        optimiser.step()
        losses.append(loss.detach())
    return [float(v) for v in losses], [float(v) for v in norms]


def points(coords, cluster_of):
    """The regression's points: one more coordinate keeps the clusters apart, as its approximation of what lies between
    clusters wants them."""
    return torch.cat([coords, 12.0 * cluster_of[:, None]], dim=1)


def main(steps=150, device="cuda:0"):
    tokens, offsets, cluster_of, y = data(1, PER, device)
    layer = Layer(0, device)
    losses, norms = fit(layer, tokens, offsets, y, steps)
    with torch.no_grad():
        coords, _, _ = layer.forward(tokens, offsets)

        probes = np.random.default_rng(1).choice([-1.0, 1.0], size=(len(y), 8))
        gp = P.Context(points(coords, cluster_of), y, np.arange(CLUSTERS + 1) * PER, probes, rank=8, device=device)
        phi, m, v = np.zeros(gp.p), np.zeros(gp.p), np.zeros(gp.p)
        nll = []
        for t in range(10):
            s = gp.nugpr_train_step(phi, m, v, t)
            phi, m, v = s["log_theta"], s["adam_m"], s["adam_v"]
            nll.append(s["nll0"])
        theta = np.exp(phi)
        gp.nugpr_build_blocks(theta)
        gp.nugpr_precond_factor()

        # held-out sequences, all but their last two tokens first
        held, off, cl, yt = data(2, 12, device)
        n = len(yt)
        whole, _, _ = layer.forward(held, off)
        ends = off[1:]
        shown = torch.ones(held.shape[0], dtype=torch.bool, device=device)
        shown[ends - 1] = shown[ends - 2] = False
        _, window, state = layer.forward(held[shown], off - 2 * torch.arange(n + 1, device=device))
        rmse = []
        for back in (2, 1):
            grown = layer.step(held[ends - back], window, state)
            rmse.append(P.binding.nugpr_rmse(gp.nugpr_predict(theta, points(grown, cl), variance=False)["mean"],
                                             yt.cpu().numpy()))
        gp.close()
    return dict(losses=losses, norms=norms, nll=nll, rmse=rmse, spread=float(yt.std()),
                apart=float((grown - whole).norm() / whole.norm()))


if __name__ == "__main__":
    out = main()
    print(f"layer: squared error {out['losses'][0]:.4f} -> {out['losses'][-1]:.4f} in {len(out['losses'])} steps, norms of the "
          f"gradients {min(out['norms']):.3f} to {max(out['norms']):.3f}")
    print(f"regression: negative log likelihood {out['nll'][0]:.2f} -> {out['nll'][-1]:.2f}")
    print(f"held-out sequences: RMSE {out['rmse'][0]:.4f} one token before their end, {out['rmse'][1]:.4f} at it "
          f"(spread of the targets {out['spread']:.4f})")
    print(f"coordinates token by token against whole sequences: {out['apart']:.1e}")
