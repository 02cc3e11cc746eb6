"""Infinities and NaN in the arrays that many channels or rows read (GPU), against autograd of the formulas in 64 bits: what is
infinite, what is NaN, and the numbers beside them, with the tolerances of test_gpu_selective_scan.py and test_gpu_short_conv.py.

All values that the sums are linear in are positive, so that infinities of two signs meet only where the formulas have both."""
import pytest
import torch

import test_gpu_selective_scan as scan
import test_gpu_short_conv as conv

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
INF, NAN = float("inf"), float("nan")


def same(got, want, tol, what, terms=None):
    got, want = got.double().cpu(), want.double().cpu()
    assert got.shape == want.shape, what
    for kind in (torch.isnan, torch.isposinf, torch.isneginf):
        assert torch.equal(kind(got), kind(want)), (what, kind.__name__, int(kind(got).sum()), int(kind(want).sum()))
    fine = torch.isfinite(want)
    bound = tol * float(want[fine].norm())
    if terms is not None:
        bound += scan.TOL[F32] * float(terms.double().cpu()[fine].norm())
    assert float((got[fine] - want[fine]).norm()) <= bound, what


def positive(lens, dim, groups, states, dtype, seed, more=True):
    """more: with a gate, D, bias and softplus."""
    v, off, dev_off, dy, ds1 = scan.inputs(lens, dim, groups, states, dtype, seed, gate=more, more=more, softplus=more)
    for k in ("x", "B", "C", "D", "z", "s0"):
        if v[k] is not None:
            v[k] = v[k].abs() + 0.25
    return v, off, dev_off, dy.abs() + 0.25, ds1.abs() + 0.25


def both(lib, v, off, dev_off, dy, ds1, clean, more=True):
    y, end = scan.forward(lib, v, dev_off, more)
    want, w_end = scan.reference(scan.double(v), off, more)
    same(y, want, scan.tolerance(y), "y")
    same(end, w_end, scan.TOL[F32], "end")
    got, g_want = scan.backward(lib, v, dev_off, dy, ds1, more), scan.wanted(v, off, dy, ds1, more)
    terms = scan.wanted(scan.magnitudes(clean), off, dy, ds1, more)
    for k in scan.NAMES:
        if v[k] is not None:
            same(got[k], g_want[k], scan.tolerance(v[k]), k, terms[k])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("states", [5, 8, 16, 24, 32, 40, 64])
@pytest.mark.parametrize("dim,groups", [(1, 1), (64, 1), (70, 1), (130, 2)])
def test_infinite_rows_of_B_and_C(lib, dim, groups, states, dtype):
    """Channels by which a group falls short of a workgroup's or a wave's are none: an infinity that they read goes nowhere."""
    v, off, dev_off, dy, ds1 = positive([37, 41], dim, groups, states, dtype, seed=dim + states)
    clean = dict(v)
    v["B"], v["C"] = v["B"].clone(), v["C"].clone()
    v["B"][11, groups - 1, states // 2] = INF          # (states are infinite from here on)
    v["C"][37 + 20, 0, states - 1] = INF               # (gradients are, back to the begin)
    both(lib, v, off, dev_off, dy, ds1, clean)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("states", [1, 5, 16, 32, 40])
@pytest.mark.parametrize("lens", [[1], [3, 5], [14], [16], [18, 31], [300]], ids=str)
def test_an_infinite_gradient_at_the_end(lib, lens, states, dtype):
    """Sequences that end amid a tile of rows: rows behind their end have no part in anything."""
    v, off, dev_off, dy, ds1 = positive(lens, 70, 1, states, dtype, seed=len(lens) + states)
    ds1[0, 3, states - 1] = ds1[-1, 65, 0] = INF
    both(lib, v, off, dev_off, dy, ds1, v)


@pytest.mark.parametrize("where", ["start", "x", "C", "end"])
@pytest.mark.parametrize("many", [0, 300])
@pytest.mark.parametrize("states,groups,dtype,more", [(1, 1, F32, True), (16, 1, F32, True), (40, 1, F32, True), (16, 2, BF16, True), (5, 3, F32, False),
                                                      (32, 2, BF16, False)])
def test_infinities_of_far_rows(lib, states, groups, dtype, more, many, where):
    """Over many rows a state's factors come to less than float32 holds, though none of them is zero: what is infinite stays so, over
    spans of 64 rows and between them.  In sequences numbered one after the other, and by their place."""
    v, off, dev_off, dy, ds1 = positive([300] + [1] * many, 6, groups, states, dtype, states, more)
    clean = dict(v)
    v["A"] = -torch.linspace(0.5, 16.0, 6 * states, device="cuda").reshape(6, states)
    if where == "start":
        v["s0"][0, 5, states - 1] = INF
    elif where == "x":
        v["x"][70, 4] = INF
    elif where == "C":
        v["C"][290, 0, 0] = INF
    else:
        ds1[0, 3, 0] = INF
    both(lib, v, off, dev_off, dy, ds1, dict(clean, A=v["A"]), more)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [INF, NAN])
@pytest.mark.parametrize("tap,width,dim", [(0, 4, 70), (1, 4, 301), (2, 3, 64), (0, 8, 33), (0, 2, 513)])
def test_weights_that_are_not_finite(lib, tap, width, dim, value, dtype):
    """A tap reaches the gradients of those rows alone that have a row so far behind them in their sequence."""
    lens = [1, 0, 2, 5, 300, 33]
    i = conv.inputs(lens, dim, width, dtype, seed=width)
    i.update({k: i[k].abs() + 0.25 for k in ("x", "w", "dy", "s0", "ds1")})
    i["w"][dim // 2, tap] = value
    got = lib.nugpr_short_conv_backward(i["x"], i["w"], i["dev_off"], i["dy"], bias=i["b"], initial_state=i["s0"], d_final_state=i["ds1"])
    want = conv.wanted(i, i["b"], False, i["s0"], i["ds1"])
    for x, w, name in zip(got, want, ("dx", "dw", "db", "ds")):
        same(x, w, conv.TOL[dtype], name)
    y, _ = lib.nugpr_short_conv_forward(i["x"], i["w"], i["dev_off"], bias=i["b"], initial_state=i["s0"])
    w, _ = conv.reference(conv.double(i["x"]), conv.double(i["w"]), conv.double(i["b"]), i["off"], False, conv.double(i["s0"]))
    same(y, w, conv.TOL[dtype], "y")
