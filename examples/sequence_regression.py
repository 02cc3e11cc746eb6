"""Regression on sequences: a layer of decayed linear attention, one low-rank adapter a cluster, makes the coordinates; the
Gaussian process regresses on them; later tokens arrive one at a time.

  1. The layer's adapters and a linear readout are fitted by gradient descent (nugpr_adapter_forward / _backward,
     nugpr_decay_attention_forward / _backward).
  2. The readout's coordinates of every sequence go into a Context: training steps, predictions for held-out sequences.
  3. Held-out sequences grow by a token each: a row through the projection, a step on the kept state
     (nugpr_decay_attention_step), a new prediction.  The same coordinates come out as from the whole sequences.

Run: python examples/sequence_regression.py"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2510_12128_amd as P  # noqa: E402

CLUSTERS, PER, WIDTH, HEADS, DIM, RANK, COORDS = 4, 256, 6, 2, 8, 2, 3


class Layer:
    """x -> [q | k | v] = x W^T + adapter, decayed attention, readout of a sequence's last row."""

    def __init__(self, seed, device):
        g = torch.Generator(device=device).manual_seed(seed)

        def r(*shape, scale):
            return torch.randn(*shape, generator=g, device=device) * scale

        out = 3 * HEADS * DIM
        self.W = r(out, WIDTH, scale=WIDTH ** -0.5)
        self.W[:2 * HEADS * DIM] = 0.0              # queries and keys look at the constant entry of a token only
        self.W[:2 * HEADS * DIM, 0] = DIM ** -0.25
        self.A = r(CLUSTERS, RANK, WIDTH, scale=0.1 * WIDTH ** -0.5)
        self.B = torch.zeros(CLUSTERS, RANK, out, device=device)
        self.R = r(HEADS * DIM, COORDS, scale=0.1 * (HEADS * DIM) ** -0.5)
        self.r = r(COORDS, scale=1.0)
        self.log_decay = torch.log(torch.tensor([0.9, 0.6], device=device))

    def trained(self):
        return [self.A, self.B, self.R, self.r]

    def split(self, qkv):
        return [t.reshape(qkv.shape[0], HEADS, DIM) for t in qkv.split(HEADS * DIM, dim=1)]     # (views)

    def forward(self, x, offsets, cluster_of):
        """Coordinates of the sequences, their end states, and what the gradient needs."""
        qkv = P.nugpr_adapter_forward(x, self.W, self.A, self.B, offsets, adapter_of=cluster_of)
        q, k, v = self.split(qkv)
        o, state = P.nugpr_decay_attention_forward(q, k, v, self.log_decay, offsets, scale=DIM ** -0.5)
        last = o[offsets[1:] - 1].reshape(-1, HEADS * DIM)
        return last @ self.R, state, (x, qkv, last)

    def backward(self, kept, offsets, cluster_of, d_coords):
        x, qkv, last = kept
        q, k, v = self.split(qkv)
        d_o = torch.zeros(x.shape[0], HEADS, DIM, device=x.device)
        d_o[offsets[1:] - 1] = (d_coords @ self.R.T).reshape(-1, HEADS, DIM)
        dq, dk, dv, _ = P.nugpr_decay_attention_backward(q, k, v, self.log_decay, offsets, d_o, scale=DIM ** -0.5)
        d_qkv = torch.cat([t.reshape(x.shape[0], -1) for t in (dq, dk, dv)], dim=1)
        _, dA, dB = P.nugpr_adapter_backward(x, self.W, self.A, self.B, offsets, d_qkv, adapter_of=cluster_of)
        return [dA, dB, last.T @ d_coords]

    def step(self, x, requests, cluster_of, state):
        """One more token of each sequence; advances the states."""
        q, k, v = self.split(P.nugpr_adapter_forward(x, self.W, self.A, self.B, requests, adapter_of=cluster_of))
        o = P.nugpr_decay_attention_step(q, k, v, self.log_decay, state, scale=DIM ** -0.5)
        return o.reshape(-1, HEADS * DIM) @ self.R


def data(seed, per, device):
    """Sequences cluster by cluster; the target of one is a decayed sum over its tokens in its cluster's own direction."""
    rng = np.random.default_rng(seed)
    along = np.random.default_rng(11).normal(size=(CLUSTERS, WIDTH)) / WIDTH ** 0.5
    tokens, targets = [], []
    for c in range(CLUSTERS):
        for _ in range(per):
            x = rng.normal(size=(int(rng.integers(4, 40)), WIDTH))
            x[:, 0] = 1.0
            w = 0.9 ** np.arange(len(x))[::-1]
            targets.append((w[:, None] * x).sum(0) @ along[c] * 0.5 + rng.normal() * 0.02)
            tokens.append(x)
    offsets = np.concatenate([[0], np.cumsum([len(x) for x in tokens])]).astype(np.int64)
    return (torch.tensor(np.concatenate(tokens), dtype=torch.float32, device=device), torch.from_numpy(offsets).to(device),
            torch.arange(CLUSTERS, dtype=torch.int32, device=device).repeat_interleave(per),
            torch.tensor(np.array(targets), dtype=torch.float32, device=device))


def fit(layer, x, offsets, cluster_of, y, steps):
    optimiser = torch.optim.Adam(layer.trained(), lr=0.01)
    losses = []
    for _ in range(steps):
        coords, _, kept = layer.forward(x, offsets, cluster_of)
        off = coords @ layer.r - y
        d = 2.0 / len(y) * off
        layer.A.grad, layer.B.grad, layer.R.grad = layer.backward(kept, offsets, cluster_of, d[:, None] * layer.r)
        layer.r.grad = coords.T @ d
        optimiser.step()
        losses.append(off.square().mean())
    return [float(v) for v in losses]


def points(coords, cluster_of):
    """The regression's points: one more coordinate keeps the clusters apart, as its approximation of what lies between
    clusters wants them."""
    return torch.cat([coords, 12.0 * cluster_of[:, None]], dim=1)


def main(steps=150, device="cuda:0"):
    x, offsets, cluster_of, y = data(1, PER, device)
    layer = Layer(0, device)
    losses = fit(layer, x, offsets, cluster_of, y, steps)
    coords, _, _ = layer.forward(x, offsets, cluster_of)

    probes = np.random.default_rng(1).choice([-1.0, 1.0], size=(len(y), 8))
    clusters = np.arange(CLUSTERS + 1) * PER
    gp = P.Context(points(coords, cluster_of), y, clusters, probes, rank=8, device=device)
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
    xt, off_t, cl_t, yt = data(2, 12, device)
    n = len(yt)
    whole, _, _ = layer.forward(xt, off_t, cl_t)
    ends = off_t[1:]
    shown = torch.ones(xt.shape[0], dtype=torch.bool, device=device)
    shown[ends - 1] = shown[ends - 2] = False
    begun = off_t - 2 * torch.arange(n + 1, device=device)
    _, state, _ = layer.forward(xt[shown], begun, cl_t)
    single = torch.arange(n + 1, device=device)
    rmse = []
    for back in (2, 1):
        grown = layer.step(xt[ends - back], single, cl_t, state)
        rmse.append(P.binding.nugpr_rmse(gp.nugpr_predict(theta, points(grown, cl_t), variance=False)["mean"],
                                         yt.cpu().numpy()))
    gp.close()
    return dict(losses=losses, nll=nll, rmse=rmse, spread=float(yt.std()), apart=float((grown - whole).norm() / whole.norm()))


if __name__ == "__main__":
    out = main()
    print(f"layer: squared error {out['losses'][0]:.4f} -> {out['losses'][-1]:.4f} in {len(out['losses'])} steps")
    print(f"regression: negative log likelihood {out['nll'][0]:.2f} -> {out['nll'][-1]:.2f}")
    print(f"held-out sequences: RMSE {out['rmse'][0]:.4f} one token before their end, {out['rmse'][1]:.4f} at it "
          f"(spread of the targets {out['spread']:.4f})")
    print(f"coordinates token by token against whole sequences: {out['apart']:.1e}")
