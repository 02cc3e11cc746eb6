"""Selective scan (GPU) against its recurrence in 64 bits, token by token; gradients by autograd of that and against
differences.

Tolerances, relative in the 2-norm.  float32: a factor e^(d A) is off by a few roundings of 2^-24 and a state forgets after
1 / (d |A|) tokens, 50 here at most, so that the factors' errors, independent of each other, add up to a few times the
root of 50; sums over 64 states, 64 channels and more, and some 1000 rows add as much.  Below 128 of 2^-24.  bfloat16 results:
rounded once, by half of 2^-7 at most, and the float32 roundings beside it are nothing.

The float32 roundings are relative to the terms that are summed, not to the sum: y of a single row without D and z is d x (B . C), and
where B . C of 64 states comes out a hundredth of a typical one, 0.1 of a norm of 8, so does y, but not its error, 2^-24 of
products of order one in a sum of order eight: 5e-5 of y.  So the bound is TOL of the result plus 128 of 2^-24 of the same sums
with the magnitudes of x, B, C, D, z, the states and the gradients given, which is never less than the terms added up."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
TOL = {F32: 128 * 2.0 ** -24, BF16: 2.0 ** -8 * 1.01}
NAMES = ("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "s0")


def reference(v, offsets, softplus):
    """y and end states of the values in v, a dict by NAMES (some None), in their type."""
    x, dt, A, B, C, D, z, bias, s0 = (v[k] for k in NAMES)
    each = x.shape[1] // B.shape[1]
    d = dt if bias is None else dt + bias
    d = torch.log1p(torch.exp(d)) if softplus else d
    ys, ends = [], []
    for s in range(len(offsets) - 1):
        h = s0[s]
        for t in range(offsets[s], offsets[s + 1]):
            b, c = B[t].repeat_interleave(each, 0), C[t].repeat_interleave(each, 0)
            h = torch.exp(d[t][:, None] * A) * h + (d[t] * x[t])[:, None] * b
            y = (c * h).sum(1)
            if D is not None:
                y = y + D * x[t]
            ys.append(y if z is None else y * z[t] * torch.sigmoid(z[t]))
        ends.append(h)
    return torch.stack(ys) if ys else x * 0.0, torch.stack(ends)


def close(x, want, tol, what="", terms=None):
    """terms: the sums of magnitudes that `want` comes from, where it may be small beside them."""
    assert x.shape == want.shape, what
    x, want = x.double().cpu(), want.double().cpu()
    err, bound = float((x - want).norm()), tol * float(want.norm())
    if terms is not None:
        bound += TOL[F32] * float(terms.norm())
    assert err <= bound or err == 0.0, (what, err / float(want.norm() + 1e-300))


def magnitudes(v):
    """The values in v, without the signs of those that the sums are linear in."""
    return {k: t if t is None or k in ("dt", "dt_bias", "A") else t.abs() for k, t in v.items()}


def odd(x):
    """The same values in rows that begin at any value."""
    wide = torch.zeros(x.shape[:-1] + (x.shape[-1] + 5,), dtype=x.dtype, device=x.device)
    wide[..., 1:1 + x.shape[-1]] = x
    return wide[..., 1:1 + x.shape[-1]]


def inputs(lens, dim, groups, states, dtype, seed=0, gate=True, more=True, softplus=True):
    gen = torch.Generator().manual_seed(seed)

    def r(*shape, t=dtype):
        return torch.randn(*shape, generator=gen).to(t).cuda()

    n = sum(lens)
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    v = dict(x=r(n, dim), B=r(n, groups, states), C=r(n, groups, states), z=r(n, dim) if gate else None,
             A=-torch.exp(torch.rand(dim, states, generator=gen) * 3.5 - 0.7).cuda(), D=r(dim, t=F32) if more else None,
             s0=r(len(lens), dim, states, t=F32))
    step = torch.exp(torch.rand(n, dim, generator=gen) * 2.5 - 3.2)        # 0.04 to 0.5
    if softplus:
        v["dt_bias"] = r(dim, t=F32) if more else None
        raw = torch.log(torch.expm1(step))
        v["dt"] = (raw - v["dt_bias"].cpu() if more else raw).to(dtype).cuda()
    else:
        v["dt"], v["dt_bias"] = step.to(dtype).cuda(), None
    return v, off, torch.from_numpy(off).cuda(), r(n, dim), r(len(lens), dim, states, t=F32)


def double(v):
    return {k: None if t is None else t.double().cpu() for k, t in v.items()}


def forward(lib, v, off, softplus=True, start=True):
    return lib.nugpr_selective_scan_forward(v["x"], v["dt"], v["A"], v["B"], v["C"], off, D=v["D"], z=v["z"],
                                            dt_bias=v["dt_bias"], softplus=softplus, initial_state=v["s0"] if start else None)


def backward(lib, v, off, dy, ds1=None, softplus=True, start=True):
    out = lib.nugpr_selective_scan_backward(v["x"], v["dt"], v["A"], v["B"], v["C"], off, dy, D=v["D"], z=v["z"],
                                            dt_bias=v["dt_bias"], softplus=softplus, initial_state=v["s0"] if start else None,
                                            d_final_state=ds1)
    return dict(zip(NAMES, out))


def wanted(v, off, dy, ds1, softplus):
    f = double(v)
    leaves = {k: t.requires_grad_() for k, t in f.items() if t is not None}
    y, end = reference(f, off, softplus)
    loss = (y * dy.double().cpu()).sum() + (0.0 if ds1 is None else (end * ds1.double().cpu()).sum())
    if not loss.requires_grad:
        return {k: torch.zeros_like(t) for k, t in leaves.items()}
    got = torch.autograd.grad(loss, list(leaves.values()), allow_unused=True)
    return {k: torch.zeros_like(t) if g is None else g for (k, t), g in zip(leaves.items(), got)}


def tolerance(t):
    return TOL[t.dtype]


LENS = [[1], [15], [16], [17], [64], [65], [0, 1, 0, 2, 129, 0, 3], [300, 7, 64, 1]]
SHAPES = [(64, 1, 16), (70, 2, 5), (130, 1, 16), (200, 4, 24), (9, 3, 1), (64, 1, 64), (100, 1, 40), (3, 1, 8), (257, 1, 13)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("dim,groups,states", SHAPES)
def test_forward(lib, lens, dim, groups, states, dtype):
    for gate, more, softplus, start in ((True, True, True, True), (False, False, False, False)):
        v, off, dev_off, _, _ = inputs(lens, dim, groups, states, dtype, len(lens) + dim, gate, more, softplus)
        y, end = forward(lib, v, dev_off, softplus, start)
        f = double(v)
        f["s0"] = f["s0"] * start
        want, w_end = reference(f, off, softplus)
        assert y.dtype == dtype and end.dtype == F32
        close(y, want, TOL[dtype], "y", reference(magnitudes(f), off, softplus)[0])
        close(end, w_end, TOL[F32], "state")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("dim,groups,states", SHAPES)
def test_backward(lib, lens, dim, groups, states, dtype):
    for gate, more, softplus, start in ((True, True, True, True), (False, False, False, False)):
        v, off, dev_off, dy, ds1 = inputs(lens, dim, groups, states, dtype, 3 * len(lens) + dim, gate, more, softplus)
        got = backward(lib, v, dev_off, dy, ds1 if start else None, softplus, start)
        if not start:
            v["s0"] = torch.zeros_like(v["s0"])
        want = wanted(v, off, dy, ds1 if start else None, softplus)
        terms = wanted(magnitudes(v), off, dy.abs(), ds1.abs() if start else None, softplus)
        for k in NAMES:
            assert (got[k] is None) == (v[k] is None), k
            if got[k] is not None:
                assert got[k].dtype == v[k].dtype
                close(got[k], want[k], tolerance(v[k]), k, terms[k])


def test_long_sequences(lib):
    """Many spans, one sequence begins inside one: the same values as the recurrence, and as the rows in one call each."""
    lens = [1500, 5, 2600]
    v, off, dev_off, dy, ds1 = inputs(lens, 40, 1, 16, F32, seed=8)
    y, end = forward(lib, v, dev_off)
    want, w_end = reference(double(v), off, True)
    close(y, want, TOL[F32])
    close(end, w_end, TOL[F32])
    got, g_want = backward(lib, v, dev_off, dy, ds1), wanted(v, off, dy, ds1, True)
    for k in NAMES:
        close(got[k], g_want[k], TOL[F32], k)


@pytest.mark.parametrize("lens", [[8400, 40, 700], [10] * 20 + [8900]], ids=["few", "many"])
def test_long_sequences_of_few_channels(lib, lens):
    """Longer spans, as their number is bounded: where that is known from the number of rows, and where it is not."""
    v, off, dev_off, dy, ds1 = inputs(lens, 6, 1, 2, F32, seed=9)
    y, end = forward(lib, v, dev_off)
    want, w_end = reference(double(v), off, True)
    close(y, want, TOL[F32])
    close(end, w_end, TOL[F32])
    got, g_want = backward(lib, v, dev_off, dy, ds1), wanted(v, off, dy, ds1, True)
    terms = wanted(magnitudes(v), off, dy.abs(), ds1.abs(), True)
    for k in NAMES:
        close(got[k], g_want[k], TOL[F32], k, terms[k])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides(lib, dtype):
    v, off, dev_off, dy, ds1 = inputs([70, 3, 130], 101, 1, 16, dtype, seed=5)
    for k in ("x", "dt", "z", "B", "C"):
        v[k] = odd(v[k])
    v["B"] = v["B"].transpose(0, 1).contiguous().transpose(0, 1)
    y, end = forward(lib, v, dev_off)
    want, w_end = reference(double(v), off, True)
    close(y, want, TOL[dtype])
    close(end, w_end, TOL[F32])
    got, g_want = backward(lib, v, dev_off, odd(dy), ds1), wanted(v, off, dy, ds1, True)
    for k in NAMES:
        close(got[k], g_want[k], tolerance(v[k]), k)


def test_one_row_of_B_for_all(lib):
    """Inputs that are one row expanded: read with a stride of zero; the gradient has a row for each."""
    v, off, dev_off, dy, ds1 = inputs([40], 64, 2, 8, F32, seed=12)
    v["B"], v["z"] = v["B"][:1].expand(40, -1, -1), v["z"][:1].expand(40, -1)
    close(forward(lib, v, dev_off)[0], reference(double(v), off, True)[0], TOL[F32])
    w = dict(v, B=v["B"].contiguous(), z=v["z"].contiguous())
    got, want = backward(lib, v, dev_off, dy, ds1), wanted(w, off, dy, ds1, True)
    for k in NAMES:
        close(got[k], want[k], TOL[F32], k)


def test_gradient_against_differences(lib):
    """Along one direction, central differences of the float64 reference with h = 1e-5: error h^2 of the third derivative and
    1e-16 / h of its roundings, below 1e-7."""
    v, off, dev_off, dy, ds1 = inputs([5, 70, 0, 20], 24, 2, 6, F32, seed=9)
    got, base = backward(lib, v, dev_off, dy, ds1), double(v)
    gen = torch.Generator().manual_seed(1)
    for k in NAMES:
        d, f = torch.randn(base[k].shape, generator=gen, dtype=torch.float64), []
        for sign in (1.0, -1.0):
            y, end = reference(dict(base, **{k: base[k] + sign * 1e-5 * d}), off, True)
            f.append(float((y * dy.double().cpu()).sum() + (end * ds1.double().cpu()).sum()))
        slope = float((got[k].double().cpu() * d).sum())
        scale = float(got[k].double().cpu().norm() * d.norm())
        assert abs(slope - (f[0] - f[1]) / 2e-5) <= TOL[F32] * scale + 1e-7 * scale, k


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim,groups,states", SHAPES)
def test_steps_go_on_where_a_prompt_ends(lib, dim, groups, states, dtype):
    lens = [9, 1, 30]
    v, off, dev_off, _, _ = inputs(lens, dim, groups, states, dtype, seed=2)
    want, end = reference(double(v), off, True)
    rows = dev_off[1:] - 1
    keep = torch.ones(sum(lens), dtype=torch.bool, device="cuda")
    keep[rows] = False
    shown = {k: t[keep] if k in ("x", "dt", "B", "C", "z") else t for k, t in v.items()}
    _, state = forward(lib, shown, dev_off - torch.arange(4, device="cuda"))
    pool = torch.randn(5, dim, states, device="cuda")
    slots = torch.tensor([4, 0, 2], dtype=torch.int32, device="cuda")
    before = pool.clone()
    pool[slots.long()] = state
    one = {k: v[k][rows] for k in ("x", "dt", "B", "C", "z")}
    y = lib.nugpr_selective_scan_step(one["x"], one["dt"], v["A"], one["B"], one["C"], pool, slots=slots, D=v["D"],
                                      z=one["z"], dt_bias=v["dt_bias"])
    close(y, want[rows.cpu()], TOL[dtype])
    close(pool[slots.long()], end, TOL[F32])
    assert torch.equal(pool[[1, 3]], before[[1, 3]])


def test_slots_of_no_request(lib):
    v, _, _, _, _ = inputs([4], 70, 1, 16, F32, gate=False, more=False, softplus=False)
    state = torch.randn(2, 70, 16, device="cuda")
    before = state.clone()
    slots = torch.tensor([1, -1, 2, 7], dtype=torch.int32, device="cuda")
    y = lib.nugpr_selective_scan_step(v["x"], v["dt"], v["A"], v["B"], v["C"], state, slots=slots, softplus=False)
    assert float(y[1:].abs().max()) == 0.0 and float(y[0].abs().max()) > 0.0
    assert torch.equal(state[0], before[0]) and not torch.equal(state[1], before[1])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_without_a_sequence(lib, dtype):
    """Rows before the first sequence and behind the last: zero, whatever they hold, and they add to no gradient."""
    v, off, dev_off, dy, ds1 = inputs([40, 25], 100, 1, 16, dtype, seed=4)
    n, front = 100, 11

    def among(t):
        wide = torch.full((n,) + t.shape[1:], float("nan"), dtype=t.dtype, device="cuda")
        wide[front:front + 65] = t
        return wide

    w = {k: among(t) if k in ("x", "dt", "B", "C", "z") else t for k, t in v.items()}
    y, end = forward(lib, w, dev_off + front)
    want, w_end = reference(double(v), off, True)
    close(y[front:front + 65], want, TOL[dtype])
    close(end, w_end, TOL[F32])
    assert float(y[:front].abs().max()) == 0.0 and float(y[front + 65:].abs().max()) == 0.0
    got, g_want = backward(lib, w, dev_off + front, among(dy), ds1), wanted(v, off, dy, ds1, True)
    for k in NAMES:
        if k in ("x", "dt", "B", "C", "z"):
            assert float(got[k][:front].abs().max()) == 0.0 and float(got[k][front + 65:].abs().max()) == 0.0, k
            got[k] = got[k][front:front + 65]
        close(got[k], g_want[k], tolerance(v[k]), k)


@pytest.mark.parametrize("states", [16, 5])
def test_a_value_that_is_not_finite_reaches_what_reads_it(lib, states):
    """An infinite x is in its channel's states from its row on, a NaN likewise; other channels and sequences are as they were."""
    lens = [200, 90]
    v, off, dev_off, _, _ = inputs(lens, 70, 1, states, F32, seed=6, gate=False)
    v["B"], v["C"] = v["B"].abs() + 0.5, v["C"].abs() + 0.5       # (no infinities of two signs)
    v["x"][37, 3], v["x"][210, 9] = float("inf"), float("nan")
    y, end = forward(lib, v, dev_off)
    want, w_end = reference(double(v), off, True)
    for got, w in ((y, want), (end, w_end)):
        got = got.double().cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(w)) and torch.equal(torch.isinf(got), torch.isinf(w))
        fine = torch.isfinite(w)
        assert float((got[fine] - w[fine]).norm()) <= TOL[F32] * float(w[fine].norm())


def test_far_steps(lib):
    """softplus far from zero on both sides, and decays that leave nothing."""
    v, off, dev_off, _, _ = inputs([64], 64, 1, 16, F32, seed=3, more=False)
    v["dt"] = torch.linspace(-60.0, 60.0, 64, device="cuda")[:, None].repeat(1, 64).contiguous()
    y, end = forward(lib, v, dev_off)
    want, w_end = reference(double(v), off, True)
    close(y, want, TOL[F32])
    close(end, w_end, TOL[F32])
    for row in range(64):                                        # rows of tiny steps are as good as the others
        close(y[row], want[row], 2 * TOL[F32], row)


def test_without_rows(lib):
    v, off, dev_off, dy, ds1 = inputs([0, 0, 0], 70, 1, 16, F32)
    y, end = forward(lib, v, dev_off)
    assert y.shape == (0, 70) and torch.equal(end, v["s0"])
    got = backward(lib, v, dev_off, dy, ds1)
    assert torch.equal(got["s0"], ds1)
    for k in ("A", "D", "dt_bias"):
        assert float(got[k].abs().max()) == 0.0
    none = torch.zeros(1, dtype=torch.int64, device="cuda")
    v["s0"] = v["s0"][:0]
    y, end = forward(lib, v, none)
    got = backward(lib, v, none, dy)
    assert end.shape == (0, 70, 16) and float(got["A"].abs().max()) == 0.0
    v, _, _, _, _ = inputs([4], 70, 1, 16, F32)
    with pytest.raises(lib.NugprError, match="no sequence"):
        forward(lib, v, none, start=False)


@pytest.mark.parametrize("states", [16, 5, 40])
@pytest.mark.parametrize("row", [36, 20, 41])
def test_gradients_where_a_value_is_not_finite(lib, states, row):
    """A NaN in a channel's x, in the last row of a sequence, amid it, or in the first: its gradients are NaN where the formulas make
    them so and the numbers they were elsewhere."""
    v, off, dev_off, dy, ds1 = inputs([37, 90], 70, 1, states, F32, seed=16)
    clean = backward(lib, v, dev_off, dy, ds1)
    v["x"][row, 3] = float("nan")
    got = backward(lib, v, dev_off, dy, ds1)
    want = wanted(v, off, dy, ds1, True)
    for k in NAMES:
        assert torch.equal(torch.isnan(got[k]).cpu(), torch.isnan(want[k])), k
        fine = ~torch.isnan(got[k])
        assert torch.equal(got[k][fine], clean[k][fine]), k


def test_rates_at_the_ends_of_their_range(lib):
    """A = 0 keeps everything, -infinity nothing; in sequences of no, one and several spans, that end amid a tile."""
    v, off, dev_off, dy, ds1 = inputs([5, 300, 0, 37], 40, 1, 8, F32, seed=21)
    v["A"][:, 0], v["A"][:, 1], v["A"][:, 2] = 0.0, float("-inf"), -1e38
    y, end = forward(lib, v, dev_off)
    want, w_end = reference(double(v), off, True)
    # (the states that keep everything are sums of 300 terms that nothing scales down)
    close(y, want, 4 * TOL[F32], "y", reference(magnitudes(double(v)), off, True)[0])
    close(end, w_end, 4 * TOL[F32], "state")
    got = backward(lib, v, dev_off, dy, ds1)
    assert all(bool(torch.isfinite(t).all()) for t in got.values())
    state = v["s0"].clone()
    y = lib.nugpr_selective_scan_step(v["x"][:4], v["dt"][:4], v["A"], v["B"][:4], v["C"][:4], state, D=v["D"], z=v["z"][:4],
                                      dt_bias=v["dt_bias"])
    one = {k: t[:4] if k in ("x", "dt", "B", "C", "z") else t for k, t in double(v).items()}
    want, w_end = reference(one, [0, 1, 2, 3, 4], True)
    close(y, want, TOL[F32])
    close(state, w_end, TOL[F32])


@pytest.mark.parametrize("many", [3, 60, 250, 1100])
def test_wide_layers(lib, many):
    """So many channels that a sequence need not be cut for want of work: alone and among sequences by the thousand, where it is.
    The reference has some of the channels, which do not read each other."""
    dim, rows, keep = 32768, 700, [0, 63, 64, 20000, 32767]
    lens = [1] * (many // 2) + [rows] + [1] * (many - many // 2)
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    dev = torch.from_numpy(off).cuda()
    gen = torch.Generator(device="cuda").manual_seed(many)

    def r(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    n = sum(lens)
    v = dict(x=r(n, dim), dt=r(n, dim) * 0.3 - 2.0, A=-torch.rand(dim, 2, generator=gen, device="cuda") - 0.2, B=r(n, 1, 2), C=r(n, 1, 2), D=r(dim),
             z=None, dt_bias=None, s0=r(len(lens), dim, 2))
    dy, ds1 = r(n, dim), r(len(lens), dim, 2)

    def some(t, k):
        if t is None or k in ("B", "C"):
            return t
        return t[:, keep] if k in ("x", "dt", "s0") else t[keep]

    few = {k: some(t, k) for k, t in v.items()}
    y, end = forward(lib, v, dev)
    want, w_end = reference(double(few), off, True)
    close(y[:, keep], want, TOL[F32], "y", reference(magnitudes(double(few)), off, True)[0])
    close(end[:, keep], w_end, TOL[F32], "state")
    got, g_want = backward(lib, v, dev, dy, ds1), wanted(few, off, dy[:, keep], ds1[:, keep], True)
    terms = wanted(magnitudes(few), off, dy[:, keep].abs(), ds1[:, keep].abs(), True)
    for k in ("x", "dt", "A", "D", "s0"):
        close(some(got[k], k), g_want[k], TOL[F32], k, terms[k])


def test_sequences_by_the_hundred(lib):
    """Equal ones, which are walked through whole, and two long ones among them, for which all are cut: the same values."""
    lens = [20] * 150 + [3000, 1200] + [20] * 90
    v, off, dev, dy, ds1 = inputs(lens, 24, 1, 4, F32, seed=33)
    y, end = forward(lib, v, dev)
    want, w_end = reference(double(v), off, True)
    close(y, want, TOL[F32], "y", reference(magnitudes(double(v)), off, True)[0])
    close(end, w_end, TOL[F32], "state")
    got, g_want = backward(lib, v, dev, dy, ds1), wanted(v, off, dy, ds1, True)
    for k in NAMES:
        close(got[k], g_want[k], TOL[F32], k)
    short = {k: t[:3000] if k in ("x", "dt", "B", "C", "z") else t[:150] if k == "s0" else t for k, t in v.items()}
    y, end = forward(lib, short, dev[:151])
    close(y, want[:3000], TOL[F32], "y")
    close(end, w_end[:150], TOL[F32], "state")
