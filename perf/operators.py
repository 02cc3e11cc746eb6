"""Operators of sequence models whose run time is tracked: linear attention with a decay for each head (over packed
sequences, its gradient, and one token at a time on kept states), and a shared projection with a low-rank adapter for each
request (and its gradient), through the entry points of `paper_2510_12128_amd`.

A case is a dict of plain values:

  kind      mix, mix_bwd (decayed linear attention over packed sequences, its gradient), mix_step (single tokens),
            adapt, adapt_bwd (projection with adapters, its gradient)
  dtype     bf16 or fp32
  seqs      sequences (mix) or requests (adapt) that the rows are cut into; mix_step: states that are kept
  rows      rows in all: tokens, or single tokens of as many requests (mix_step)
  ragged    lengths: 0 equal, else spread over their logarithm from one row up, every seventh sequence empty, by this seed
  heads, kv, dk, dv    query heads, key / value heads, widths
  fused     query, key and value are slices of one buffer, as one projection writes them
  state     the sequences go on from given states, and the states' gradients are given too
  inp, out, rank, adapters    widths of the projection, rank and number of the adapters
"""
import math

import numpy as np
import torch

own = False

_DEFAULTS = dict(dtype="bf16", seqs=1, rows=1, ragged=0, heads=0, kv=0, dk=0, dv=0, fused=False, state=False, inp=0, out=0,
                 rank=0, adapters=0)
CHUNK = 64                     # rows of a block of the plain form


def _case(name, **kw):
    c = dict(_DEFAULTS)
    c.update(kw)
    return dict(c, name=name)


def listed():
    return [
        # A prompt of ordinary length: few heads, so its length has to be split to fill the card.
        _case("mix_prompt", kind="mix", rows=2048, heads=8, kv=8, dk=64, dv=64, fused=True),
        # The longest document: shared key / value heads, memory traffic and arithmetic about balanced.
        _case("mix_long", kind="mix", rows=65536, heads=16, kv=4, dk=128, dv=128),
        # Sequences of very different lengths, empty ones among them, in the framework's own storage type, continued.
        _case("mix_packed_fp32", kind="mix", dtype="fp32", seqs=40, rows=20011, ragged=3, heads=8, kv=8, dk=64, dv=64,
              fused=True, state=True),
        # The gradient in training: a batch of equal sequences.
        _case("mix_bwd_train", kind="mix_bwd", seqs=16, rows=16384, heads=16, kv=16, dk=128, dv=128),
        # The gradient at odd widths, shared heads, uneven lengths, with gradients of the states.
        _case("mix_bwd_odd_fp32", kind="mix_bwd", dtype="fp32", seqs=9, rows=5003, ragged=5, heads=6, kv=2, dk=40, dv=72,
              state=True),
        # One new token of one sequence: latency.
        _case("mix_step_one", kind="mix_step", seqs=1, rows=1, heads=8, kv=8, dk=64, dv=64),
        # One new token of each of many sequences: the traffic of the states.
        _case("mix_step_many", kind="mix_step", seqs=300, rows=256, heads=16, kv=16, dk=128, dv=128),
        # Single tokens of two dozen requests, eight adapters between them: the traffic of the weights.
        _case("adapt_tokens", kind="adapt", seqs=24, rows=24, inp=2048, out=2048, rank=16, adapters=8),
        # Prompts of sixteen requests: a large matrix product.
        _case("adapt_prompt", kind="adapt", seqs=16, rows=8192, ragged=7, inp=4096, out=4096, rank=16, adapters=12),
        # Features of 32768 points in 32 clusters, one adapter a cluster, as the regression takes them (20 dimensions).
        _case("adapt_features_fp32", kind="adapt", dtype="fp32", seqs=32, rows=32768, inp=512, out=20, rank=4, adapters=32),
        # The gradient in training.
        _case("adapt_bwd_train", kind="adapt_bwd", seqs=8, rows=4096, inp=2048, out=2048, rank=16, adapters=8),
        # The gradient at odd widths, with requests that share adapters.
        _case("adapt_bwd_odd_fp32", kind="adapt_bwd", dtype="fp32", seqs=13, rows=1501, ragged=9, inp=500, out=301, rank=5,
              adapters=4),
    ]


def draw(rng):
    """Another case of the same ranges: any kind and type, lengths, widths and numbers of heads over their logarithm, odd
    ones among them, equal and uneven sequences."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["mix", "mix_bwd", "mix_step", "adapt", "adapt_bwd"])
    c = dict(_DEFAULTS, kind=kind, dtype=rng.choice(["bf16", "bf16", "fp32"]), ragged=rng.choice([0, 1 + rng.randrange(1000)]))
    if kind.startswith("mix"):
        c["kv"] = rng.choice([1, 2, 3, 4, 8, 12, 16])
        c["heads"] = c["kv"] * rng.choice([1, 1, 2, 4])
        c["dk"] = rng.choice([16, 32, 40, 64, 64, 80, 96, 128, 128])
        c["dv"] = rng.choice([c["dk"], c["dk"], 24, 64, 100, 128])
        c["fused"] = c["dk"] == c["dv"] and rng.random() < 0.5
        c["state"] = rng.random() < 0.5
        if kind == "mix_step":
            c["rows"] = log(1, 256)
            c["seqs"] = c["rows"] + rng.randrange(20)
            c["ragged"] = 0
        else:
            c["rows"] = log(64, 65536 if kind == "mix" else 16384)
            while c["rows"] * c["heads"] > (1 << 20 if kind == "mix" else 1 << 18):
                c["rows"] = c["rows"] * 3 // 4
            c["seqs"] = log(1, max(1, min(128, c["rows"] // 16)))
            c["rows"] = c["rows"] if c["ragged"] else c["rows"] // c["seqs"] * c["seqs"]
    else:
        c["inp"] = rng.choice([log(64, 4096), 64 * log(1, 64)])
        c["out"] = rng.choice([log(8, 4096), 64 * log(1, 64)])
        c["rank"] = rng.choice([1, 4, 5, 8, 16, 16, 32, 64])
        c["rows"] = log(1, 8192)
        while c["rows"] * c["inp"] * c["out"] * (4 if c["dtype"] == "fp32" or kind == "adapt_bwd" else 1) > 1 << 37:
            c["rows"] = c["rows"] * 3 // 4
        c["seqs"] = log(1, min(64, c["rows"]))
        c["adapters"] = rng.choice([c["seqs"], max(1, c["seqs"] // 2)])
        c["rows"] = c["rows"] if c["ragged"] else c["rows"] // c["seqs"] * c["seqs"]
    if 3072 in c.values():
        c = {k: 3056 if v == 3072 else v for k, v in c.items()}
    return c


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _offsets(c):
    """Where the sequences begin in the rows."""
    n, s = c["rows"], c["seqs"]
    if not c["ragged"]:
        return np.arange(s + 1, dtype=np.int64) * (n // s)
    rng = np.random.default_rng(c["ragged"])
    raw = np.exp(rng.uniform(0.0, 5.0, size=s))
    if s > 7:
        raw[6::7] = 0.0
    return np.concatenate([[0], np.round(np.cumsum(raw) / raw.sum() * n)]).astype(np.int64)


def _type(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def prepare(c, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(7919 * (seed + 1) + 3)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device=dev) * scale).to(_type(c))

    n = c["rows"]
    s = dict(kind=c["kind"], rows=n)
    if c["kind"].startswith("mix"):
        h, kv, dk, dv = c["heads"], c["kv"], c["dk"], c["dv"]
        if c["fused"]:
            every = normal(n, h + 2 * kv, dk)
            s["q"], s["k"], s["v"] = every[:, :h], every[:, h:h + kv], every[:, h + kv:]
        else:
            s["q"], s["k"], s["v"] = normal(n, h, dk), normal(n, kv, dk), normal(n, kv, dv)
        s["scale"] = dk ** -0.5
        # decays from 1 - 1/16 to 1 - 1/4096, one a head that keeps a state
        s["log_decay"] = torch.log1p(-2.0 ** -torch.linspace(4, 12, kv, device=dev, dtype=torch.float64)).float()
        if c["kind"] == "mix_step":
            s["state"] = torch.randn(c["seqs"], kv, dk, dv, generator=g, device=dev)
            s["slots"] = torch.randperm(c["seqs"], generator=g, device=dev)[:n].int()
            return s
        s["initial_state"] = torch.randn(c["seqs"], kv, dk, dv, generator=g, device=dev) if c["state"] else None
        if c["kind"] == "mix_bwd":
            s["d_out"] = normal(n, h, dv)
            s["d_final_state"] = torch.randn(c["seqs"], kv, dk, dv, generator=g, device=dev) if c["state"] else None
        o = _offsets(c)
        s["offsets"] = torch.from_numpy(o).to(dev)
        s["blocks"] = int(np.sum(-(-np.diff(o) // CHUNK)))
        return s
    s["x"] = normal(n, c["inp"])
    s["W"] = normal(c["out"], c["inp"], scale=c["inp"] ** -0.5)
    s["A"] = normal(c["adapters"], c["rank"], c["inp"], scale=c["inp"] ** -0.5)
    s["B"] = normal(c["adapters"], c["rank"], c["out"], scale=0.5 * c["rank"] ** -0.5)
    s["scale"] = 2.0
    s["offsets"] = torch.from_numpy(_offsets(c)).to(dev)
    s["adapter_of"] = torch.randint(0, c["adapters"], (c["seqs"],), generator=g, device=dev, dtype=torch.int32)
    if c["kind"] == "adapt_bwd":
        s["d_out"] = normal(n, c["out"])
    return s


# ---- the calls ------------------------------------------------------------------------------------------------------
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    import paper_2510_12128_amd as P
    kind = s["kind"]
    if kind == "mix":
        return P.nugpr_decay_attention_forward(s["q"], s["k"], s["v"], s["log_decay"], s["offsets"], scale=s["scale"],
                                               initial_state=s["initial_state"])
    if kind == "mix_bwd":
        return P.nugpr_decay_attention_backward(s["q"], s["k"], s["v"], s["log_decay"], s["offsets"], s["d_out"],
                                                scale=s["scale"], initial_state=s["initial_state"],
                                                d_final_state=s["d_final_state"])
    if kind == "mix_step":
        o = P.nugpr_decay_attention_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"], slots=s["slots"],
                                         scale=s["scale"])
        return o, s["state"]
    if kind == "adapt":
        return P.nugpr_adapter_forward(s["x"], s["W"], s["A"], s["B"], s["offsets"], adapter_of=s["adapter_of"],
                                       scale=s["scale"])
    return P.nugpr_adapter_backward(s["x"], s["W"], s["A"], s["B"], s["offsets"], s["d_out"], adapter_of=s["adapter_of"],
                                    scale=s["scale"])


# ---- the plain forms ------------------------------------------------------------------------------------------------
def _plain(s):
    kind = s["kind"]
    if kind == "mix_step":
        return _plain_step(s)
    if kind.startswith("adapt"):
        return _plain_adapt(s)
    q, k, v = s["q"].float() * s["scale"], s["k"].float(), s["v"].float()
    g, kv = q.shape[1] // k.shape[1], k.shape[1]
    decay = s["log_decay"].repeat_interleave(g)
    k, v = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
    S0 = None if s["initial_state"] is None else s["initial_state"].repeat_interleave(g, 1)
    if kind == "mix":
        o, S = _scan(q, k, v, decay, s["offsets"], s["blocks"], S0, False)
        return o.to(s["q"].dtype), S[:, ::g].contiguous()
    do = s["d_out"].float()
    # the gradients are scans of the same kind: over v, k with the roles exchanged, and backwards in time
    dq, _ = _scan(do, v, k, decay, s["offsets"], s["blocks"], None if S0 is None else S0.transpose(2, 3), False)
    R = None
    if s["d_final_state"] is not None:      # counted once for the heads that share it
        R = torch.zeros(S0.shape, device=S0.device)
        R[:, ::g] = s["d_final_state"]
    dv, dS = _scan(k, q, do, decay, s["offsets"], s["blocks"], R, True)
    dk, _ = _scan(v, do, q, decay, s["offsets"], s["blocks"], None if R is None else R.transpose(2, 3), True)
    n = q.shape[0]
    t = s["q"].dtype
    return ((dq * s["scale"]).to(t), dk.reshape(n, kv, g, -1).sum(2).to(t), dv.reshape(n, kv, g, -1).sum(2).to(t),
            dS.reshape(dS.shape[0], kv, g, dS.shape[2], dS.shape[3]).sum(2))


def _scan(q, k, v, decay, offsets, blocks, S0, back):
    """o_t = q_t S_t, S_t = e^decay S_t-1 + k_t v_t^T over each sequence, in blocks of CHUNK rows: a product inside each
    block, one of the block's start state, and one over the blocks that gives all start states.  back: against time, and
    the state takes its decay before it is read, not after."""
    e, n, dev = (1 if back else 0), q.shape[0], q.device
    lens = offsets[1:] - offsets[:-1]
    each = (lens + CHUNK - 1) // CHUNK
    seq = torch.repeat_interleave(torch.arange(lens.numel(), device=dev), each, output_size=blocks)
    number = torch.arange(blocks, device=dev) - (torch.cumsum(each, 0) - each)[seq]
    i = torch.arange(CHUNK, device=dev)
    at = number[:, None] * CHUNK + i
    live = at < lens[seq][:, None]
    count = live.sum(1)
    row = torch.where(live, offsets[seq + 1][:, None] - 1 - at if back else offsets[seq][:, None] + at, 0)

    def cut(x):                             # rows x heads x width -> blocks x heads x CHUNK x width
        return (x[row] * live[:, :, None, None]).permute(0, 2, 1, 3)

    q, k, v = cut(q), cut(k), cut(v)
    apart = i[:, None] - i[None, :]
    inside = torch.exp(decay[:, None, None] * apart.clamp(min=0)) * (apart >= 0)
    o = torch.matmul(torch.matmul(q, k.transpose(2, 3)) * inside, v)
    left = (count[:, None] - 1 + e - i[None, :]).clamp(min=0)
    kw = k * torch.exp(decay[None, :, None] * left[:, None, :])[..., None]
    local = torch.matmul(kw.transpose(2, 3), v)
    h, a, b = local.shape[1:]
    between = CHUNK * (number[:, None] - number[None, :] - 1)
    before = (seq[:, None] == seq[None, :]) & (between >= 0)
    carry = torch.exp(decay[:, None, None] * between.clamp(min=0)) * before
    start = torch.matmul(carry, local.transpose(0, 1).reshape(h, blocks, a * b)).reshape(h, blocks, a, b).transpose(0, 1)
    if S0 is not None:
        start = start + S0[seq] * torch.exp(decay[None, :] * (CHUNK * number)[:, None])[..., None, None]
    o = o + torch.matmul(q, start) * torch.exp(decay[:, None] * (i[None, :] + 1 - e))[None, :, :, None]
    out = torch.zeros(n + 1, h, b, device=dev)          # the last row takes what lies behind the ends
    out.index_put_((torch.where(live, row, n).reshape(-1),), o.permute(0, 2, 1, 3).reshape(-1, h, b))
    S = torch.zeros(lens.numel() + 1, h, a, b, device=dev)
    if S0 is not None:
        S[:-1] = S0
    end = start * torch.exp(decay[None, :] * count[:, None])[..., None, None] + local
    S.index_put_((torch.where(number == each[seq] - 1, seq, lens.numel()),), end)
    return out[:-1], S[:-1]


def _plain_step(s):
    q, k, v = s["q"].float() * s["scale"], s["k"].float(), s["v"].float()
    slots = s["slots"].long()
    kv = k.shape[1]
    S = s["state"][slots] * torch.exp(s["log_decay"])[None, :, None, None] + k[..., :, None] * v[..., None, :]
    s["state"][slots] = S
    o = torch.matmul(q.reshape(q.shape[0], kv, -1, q.shape[2]), S).reshape(q.shape[0], q.shape[1], -1)
    return o.to(s["q"].dtype), s["state"]


def _plain_adapt(s):
    x, W, t = s["x"].float(), s["W"].float(), s["x"].dtype
    na, r, inp = s["A"].shape
    A, B = s["A"].float().reshape(na * r, inp), s["B"].float().reshape(na * r, -1)
    # every adapter on every row, then the row's own one
    seq = torch.repeat_interleave(s["adapter_of"].long(), s["offsets"][1:] - s["offsets"][:-1], output_size=s["rows"])
    mine = (seq[:, None] == torch.arange(na, device=x.device)).repeat_interleave(r, 1) * s["scale"]
    H = torch.matmul(x, A.T) * mine
    if s["kind"] == "adapt":
        return (torch.matmul(x, W.T) + torch.matmul(H, B)).to(t)
    dy = s["d_out"].float()
    G = torch.matmul(dy, B.T) * mine
    dx = torch.matmul(dy, W) + torch.matmul(G, A)
    return dx.to(t), torch.matmul(G.T, x).reshape(na, r, -1).to(t), torch.matmul(H.T, dy).reshape(na, r, -1).to(t)


# ---- from the definitions, in 64 bits -------------------------------------------------------------------------------
def exact(c, seed):
    s = prepare(c, seed)
    f = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if c["kind"] == "mix_step":
        S, o = f["state"].clone(), torch.zeros(c["rows"], c["heads"], c["dv"], dtype=torch.float64, device="cuda:0")
        lam = torch.exp(f["log_decay"])
        for b, slot in enumerate(s["slots"].tolist()):
            for h in range(c["heads"]):
                j = h // (c["heads"] // c["kv"])
                now = lam[j] * f["state"][slot, j] + torch.outer(f["k"][b, j], f["v"][b, j])
                o[b, h] = s["scale"] * (f["q"][b, h] @ now)
                S[slot, j] = now
        return o, S
    off = s["offsets"].tolist()
    if c["kind"].startswith("adapt"):
        return _exact_adapt(c, s, f, off)
    q, k, v, n = f["q"] * s["scale"], f["k"], f["v"], c["rows"]
    grad = c["kind"] == "mix_bwd"
    dev = q.device
    o = torch.zeros(n, c["heads"], c["dv"], dtype=torch.float64, device=dev)
    S = torch.zeros(c["seqs"], c["kv"], c["dk"], c["dv"], dtype=torch.float64, device=dev)
    dq, dk, dv, dS = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v), torch.zeros_like(S)
    for b in range(c["seqs"]):
        lo, hi = off[b], off[b + 1]
        L = hi - lo
        t = torch.arange(L, device=dev, dtype=torch.float64)
        for h in range(c["heads"]):
            j = h // (c["heads"] // c["kv"])
            g = f["log_decay"][j]
            first = h % (c["heads"] // c["kv"]) == 0
            K, V, Q = k[lo:hi, j], v[lo:hi, j], q[lo:hi, h]
            S0 = f["initial_state"][b, j] if c["state"] else torch.zeros_like(S[b, j])
            if first and not grad:
                S[b, j] = torch.exp(g * L) * S0 + (K * torch.exp(g * (L - 1 - t))[:, None]).T @ V
            if first and grad and c["state"]:
                R = f["d_final_state"][b, j]
                w = torch.exp(g * (L - 1 - t))[:, None]
                dk[lo:hi, j] += w * (V @ R.T)
                dv[lo:hi, j] += w * (K @ R)
                dS[b, j] += torch.exp(g * L) * R
            if grad:
                dO = f["d_out"][lo:hi, h]
                dS[b, j] += (Q * torch.exp(g * (t + 1))[:, None]).T @ dO
            for r0 in range(0, L, 2048):
                r1 = min(L, r0 + 2048)
                apart = t[r0:r1, None] - t[None, :r1]
                D = torch.exp(g * apart.clamp(min=0)) * (apart >= 0)
                w = torch.exp(g * (t[r0:r1] + 1))[:, None]
                P = (Q[r0:r1] @ K[:r1].T) * D
                if not grad:
                    o[lo + r0:lo + r1, h] = P @ V[:r1] + w * (Q[r0:r1] @ S0)
                    continue
                dP = (dO[r0:r1] @ V[:r1].T) * D
                dq[lo + r0:lo + r1, h] = s["scale"] * (dP @ K[:r1] + w * (dO[r0:r1] @ S0.T))
                dk[lo:lo + r1, j] += dP.T @ Q[r0:r1]
                dv[lo:lo + r1, j] += P.T @ dO[r0:r1]
    return (dq, dk, dv, dS) if grad else (o, S)


def _exact_adapt(c, s, f, off):
    y = f["x"] @ f["W"].T
    grad = c["kind"] == "adapt_bwd"
    dx = f["d_out"] @ f["W"] if grad else None
    dA, dB = torch.zeros_like(f["A"]), torch.zeros_like(f["B"])
    for b, a in enumerate(s["adapter_of"].tolist()):
        rows = slice(off[b], off[b + 1])
        low = f["x"][rows] @ f["A"][a].T
        y[rows] += s["scale"] * (low @ f["B"][a])
        if grad:
            up = f["d_out"][rows] @ f["B"][a].T
            dx[rows] += s["scale"] * (up @ f["A"][a])
            dA[a] += s["scale"] * (up.T @ f["x"][rows])
            dB[a] += s["scale"] * (low.T @ f["d_out"][rows])
    return (dx, dA, dB) if grad else y


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(c):
    size, n = (2 if c["dtype"] == "bf16" else 4), c["rows"]
    if c["kind"].startswith("mix"):
        h, kv, dk, dv = c["heads"], c["kv"], c["dk"], c["dv"]
        qkvo = size * n * (h * dk + kv * dk + kv * dv + h * dv)
        state = 4 * kv * dk * dv
        one = 2.0 * n * dk * dv             # an update of a state, or a product with one, for every row
        if c["kind"] == "mix_step":
            return {"bytes": qkvo + 2 * n * state, "flops": one * (h + kv)}
        given = 1 if c["state"] else 0
        if c["kind"] == "mix":
            return {"bytes": qkvo + c["seqs"] * state * (1 + given), "flops": one * (h + kv)}
        return {"bytes": qkvo + size * n * (h * dk + kv * dk + kv * dv) + c["seqs"] * state * (1 + 2 * given),
                "flops": one * (2 * h + 3 * kv)}
    inp, out, r = c["inp"], c["out"], c["rank"]
    used = min(c["adapters"], c["seqs"])
    low = 2.0 * n * r * (inp + out)
    if c["kind"] == "adapt":
        return {"bytes": size * (n * (inp + out) + inp * out + used * r * (inp + out)), "flops": 2.0 * n * inp * out + low}
    return {"bytes": size * (n * (2 * inp + out) + inp * out + (used + c["adapters"]) * r * (inp + out)),
            "flops": 2.0 * n * inp * out + 2 * low + 2.0 * n * r * inp}
