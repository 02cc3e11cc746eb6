"""Short causal convolution (GPU) against its sums in 64 bits, gradients by autograd of those and against differences.

Tolerances, relative in the 2-norm.  float32: sums of up to nine products, of some 1000 rows for the weights, and a handful of
roundings more in the sigmoid, each 2^-24 and independent of the others: below 64 of them.  bfloat16 results: rounded once,
by half of 2^-7 at most, and the float32 roundings beside it are nothing."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
TOL = {F32: 64 * 2.0 ** -24, BF16: 2.0 ** -8}


def reference(x, w, b, offsets, silu, window):
    """In the type of the inputs: y and the windows at the sequences' end."""
    W = w.shape[1]
    ys, ends = [], []
    for s in range(len(offsets) - 1):
        every = torch.cat([window[s], x[offsets[s]:offsets[s + 1]]])
        n = every.shape[0] - (W - 1)
        p = sum(w[:, j] * every[j:j + n] for j in range(W)) + (0.0 if b is None else b)
        ys.append(p * torch.sigmoid(p) if silu else p)
        ends.append(every[n:])
    return torch.cat(ys), torch.stack(ends)


def close(x, want, tol, what=""):
    assert x.shape == want.shape, what
    x, want = x.double().cpu(), want.double().cpu()
    err = float((x - want).norm())
    assert err <= tol * float(want.norm()) or err == 0.0, (what, err / float(want.norm() + 1e-300))


def place(x, dtype, layout="dense"):
    x = x.to(dtype).cuda()
    if layout == "dense":
        return x
    wide = torch.zeros(x.shape[0], x.shape[1] + 5, dtype=dtype, device="cuda")     # rows that begin at any value
    wide[:, 1:1 + x.shape[1]] = x
    return wide[:, 1:1 + x.shape[1]]


def inputs(lens, dim, width, dtype, seed=0, layout="dense"):
    gen = torch.Generator().manual_seed(seed)

    def r(*shape):
        return torch.randn(*shape, generator=gen)

    n = sum(lens)
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    return dict(x=place(r(n, dim), dtype, layout), w=place(r(dim, width) * width ** -0.5, dtype), b=place(r(1, dim), dtype)[0],
                dy=place(r(n, dim), dtype, layout), off=off, dev_off=torch.from_numpy(off).cuda(),
                s0=r(len(lens), width - 1, dim).to(dtype).cuda(), ds1=r(len(lens), width - 1, dim).to(dtype).cuda())


def double(t):
    return t.double().cpu()


LENS = [[1], [2], [7], [8], [33], [0, 1, 0, 2, 129, 0, 3], [300, 7, 64, 1], [1100]]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("dim,width", [(64, 4), (301, 3), (513, 2), (5, 8), (1024, 4), (20, 1), (257, 5), (96, 6), (33, 7)])
@pytest.mark.parametrize("silu", [False, True])
def test_forward(lib, lens, dim, width, silu, dtype):
    i = inputs(lens, dim, width, dtype, seed=len(lens) + dim)
    for start, bias in ((None, None), (i["s0"], i["b"])):
        y, end = lib.nugpr_short_conv_forward(i["x"], i["w"], i["dev_off"], bias=bias, silu=silu, initial_state=start)
        want, w_end = reference(double(i["x"]), double(i["w"]), None if bias is None else double(bias), i["off"], silu,
                                double(i["s0"]) * (start is not None))
        assert y.dtype == dtype and end.dtype == dtype
        close(y, want, TOL[dtype], "y")
        assert torch.equal(end.double().cpu(), w_end)


def wanted(i, bias, silu, start, d_end):
    leaves = [double(i["x"]), double(i["w"]), double(i["b"]), double(i["s0"]) * (start is not None)]
    for t in leaves:
        t.requires_grad_()
    x, w, b, s0 = leaves
    y, end = reference(x, w, b if bias is not None else None, i["off"], silu, s0)
    loss = (y * double(i["dy"])).sum() + (0.0 if d_end is None else (end * double(d_end)).sum())
    return torch.autograd.grad(loss, leaves, allow_unused=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("dim,width", [(64, 4), (301, 3), (513, 2), (5, 8), (1024, 4), (20, 1), (257, 5), (96, 6), (33, 7)])
@pytest.mark.parametrize("silu", [False, True])
def test_backward(lib, lens, dim, width, silu, dtype):
    i = inputs(lens, dim, width, dtype, seed=3 * len(lens) + dim)
    for start, end, bias in ((None, None, None), (i["s0"], i["ds1"], i["b"])):
        dx, dw, db, ds = lib.nugpr_short_conv_backward(i["x"], i["w"], i["dev_off"], i["dy"], bias=bias, silu=silu,
                                                       initial_state=start, d_final_state=end)
        gx, gw, gb, gs = wanted(i, bias, silu, start, end)
        close(dx, gx, TOL[dtype], "dx")
        close(dw, gw, TOL[dtype], "dw")
        assert (db is None) == (bias is None)
        if db is not None:
            close(db, gb, TOL[dtype], "db")
        close(ds, torch.zeros_like(double(ds)) if gs is None else gs, TOL[dtype], "ds")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides(lib, dtype):
    i = inputs([70, 3, 130], 101, 4, dtype, seed=5, layout="odd")
    y, _ = lib.nugpr_short_conv_forward(i["x"], i["w"], i["dev_off"], bias=i["b"], silu=True, initial_state=i["s0"])
    close(y, reference(double(i["x"]), double(i["w"]), double(i["b"]), i["off"], True, double(i["s0"]))[0], TOL[dtype])
    got = lib.nugpr_short_conv_backward(i["x"], i["w"], i["dev_off"], i["dy"], bias=i["b"], silu=True, initial_state=i["s0"],
                                        d_final_state=i["ds1"])
    for x, want, name in zip(got, wanted(i, i["b"], True, i["s0"], i["ds1"]), ("dx", "dw", "db", "ds")):
        close(x, want, TOL[dtype], name)
    one = i["x"][:1].expand(3, -1)                              # one row for three requests
    state = i["s0"].clone()
    y = lib.nugpr_short_conv_step(one, i["w"], state, bias=i["b"])
    want, end = reference(double(one), double(i["w"]), double(i["b"]), [0, 1, 2, 3], False, double(i["s0"]))
    close(y, want, TOL[dtype])
    assert torch.equal(double(state), end)


def test_gradient_against_differences(lib):
    """Along one direction, central differences of the float64 reference with h = 1e-5: error h^2 of the third derivative,
    below 1e-9 of values of order one, and 1e-16 / h from its roundings."""
    i = inputs([5, 70, 0, 2], 24, 4, F32, seed=9)
    got = lib.nugpr_short_conv_backward(i["x"], i["w"], i["dev_off"], i["dy"], bias=i["b"], silu=True, initial_state=i["s0"],
                                        d_final_state=i["ds1"])
    base = [double(i[k]) for k in ("x", "w", "b", "s0")]
    gen = torch.Generator().manual_seed(1)
    for which, name in enumerate(("x", "w", "b", "s0")):
        d, f = torch.randn(base[which].shape, generator=gen, dtype=torch.float64), []
        for sign in (1.0, -1.0):
            at = [b + sign * 1e-5 * d if j == which else b for j, b in enumerate(base)]
            y, end = reference(at[0], at[1], at[2], i["off"], True, at[3])
            f.append(float((y * double(i["dy"])).sum() + (end * double(i["ds1"])).sum()))
        slope = float((double(got[which]) * d).sum())
        scale = float(double(got[which]).norm() * d.norm())
        assert abs(slope - (f[0] - f[1]) / 2e-5) <= TOL[F32] * scale + 1e-7 * abs(slope), name


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim,width", [(64, 4), (301, 3), (7, 8), (40, 1)])
def test_steps_go_on_where_a_prompt_ends(lib, dim, width, dtype):
    """A prompt, then single tokens: the same values as the whole sequences give."""
    lens = [9, 1, 30]
    i = inputs(lens, dim, width, dtype, seed=2)
    whole, end = lib.nugpr_short_conv_forward(i["x"], i["w"], i["dev_off"], bias=i["b"], silu=True)
    first = [n - 1 for n in lens]
    shown = torch.cat([i["x"][i["off"][s]:i["off"][s] + first[s]] for s in range(3)])
    off = torch.tensor(np.concatenate([[0], np.cumsum(first)]), device="cuda")
    _, state = lib.nugpr_short_conv_forward(shown, i["w"], off, bias=i["b"], silu=True)
    order = torch.tensor([2, 0, 1])
    pool = torch.randn(5, width - 1, dim, device="cuda").to(dtype)
    slots = torch.tensor([4, 0, 2], dtype=torch.int32, device="cuda")
    before = pool.clone()
    pool[slots.long()] = state[order.cuda()]
    last = i["x"][i["dev_off"][1:] - 1][order.cuda()]
    y = lib.nugpr_short_conv_step(last, i["w"], pool, slots=slots, bias=i["b"], silu=True)
    assert torch.equal(y, whole[i["dev_off"][1:] - 1][order.cuda()])
    assert torch.equal(pool[slots.long()], end[order.cuda()])
    assert torch.equal(pool[[1, 3]], before[[1, 3]])


def test_slots_of_no_request(lib):
    i = inputs([4], 70, 4, F32)
    state = torch.randn(2, 3, 70, device="cuda")
    before = state.clone()
    slots = torch.tensor([1, -1, 2, 7], dtype=torch.int32, device="cuda")
    y = lib.nugpr_short_conv_step(i["x"], i["w"], state, slots=slots, bias=i["b"])
    assert float(y[1:].abs().max()) == 0.0 and float(y[0].abs().max()) > 0.0
    assert torch.equal(state[0], before[0]) and not torch.equal(state[1], before[1])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_without_a_sequence(lib, dtype):
    """Rows before the first sequence and behind the last: zero, whatever they hold, and they add to no gradient."""
    i = inputs([40, 25], 100, 4, dtype, seed=4)
    n, front = 100, 11
    x, dy = (torch.full((n, 100), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    x[front:front + 65], dy[front:front + 65] = i["x"], i["dy"]
    off = i["dev_off"] + front
    y, end = lib.nugpr_short_conv_forward(x, i["w"], off, bias=i["b"], silu=True)
    want, w_end = lib.nugpr_short_conv_forward(i["x"], i["w"], i["dev_off"], bias=i["b"], silu=True)
    close(y[front:front + 65], want, 0.0)
    assert torch.equal(end, w_end)
    assert float(y[:front].abs().max()) == 0.0 and float(y[front + 65:].abs().max()) == 0.0
    dx, dw, db, _ = lib.nugpr_short_conv_backward(x, i["w"], off, dy, bias=i["b"], silu=True)
    gx, gw, gb, _ = lib.nugpr_short_conv_backward(i["x"], i["w"], i["dev_off"], i["dy"], bias=i["b"], silu=True)
    assert torch.equal(dx[front:front + 65], gx)
    assert float(dx[:front].abs().max()) == 0.0 and float(dx[front + 65:].abs().max()) == 0.0
    close(dw, gw, 2 * TOL[dtype])                              # (other rows a wave: sums in another order)
    close(db, gb, 2 * TOL[dtype])


def test_a_value_that_is_not_finite_reaches_what_reads_it(lib):
    i = inputs([20, 20], 40, 4, F32, seed=6)
    x = i["x"].clone()
    x[5, 3], x[30, 9] = float("inf"), float("nan")
    y, _ = lib.nugpr_short_conv_forward(x, i["w"], i["dev_off"], bias=i["b"])
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[5:9, 3] = want[30:34, 9] = True
    assert torch.equal(bad, want)


def test_without_rows_or_sequences(lib):
    w, b = torch.randn(6, 4, device="cuda"), torch.randn(6, device="cuda")
    x = torch.zeros(0, 6, device="cuda")
    s0 = torch.randn(3, 3, 6, device="cuda")
    off = torch.zeros(4, dtype=torch.int64, device="cuda")
    y, end = lib.nugpr_short_conv_forward(x, w, off, bias=b, initial_state=s0)
    assert y.shape == (0, 6) and torch.equal(end, s0)
    dx, dw, db, ds = lib.nugpr_short_conv_backward(x, w, off, x, bias=b, d_final_state=s0)
    assert torch.equal(ds, s0) and float(dw.abs().max()) == 0.0 and float(db.abs().max()) == 0.0
    none = torch.zeros(1, dtype=torch.int64, device="cuda")
    rows = torch.randn(9, 6, device="cuda")
    y, end = lib.nugpr_short_conv_forward(rows, w, none)
    assert float(y.abs().max()) == 0.0 and end.shape == (0, 3, 6)
    dx, dw, _, ds = lib.nugpr_short_conv_backward(rows, w, none, rows)
    assert float(dx.abs().max()) == 0.0 and float(dw.abs().max()) == 0.0
