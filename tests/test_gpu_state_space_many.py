"""Hundreds of sequences of which some are cut into spans (GPU): values and gradients of all against the recurrence in 64 bits."""
import numpy as np
import pytest
import torch

import test_gpu_selective_scan as scan
import test_gpu_short_conv as conv

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
LENS = {
    # spans of 64 rows: one, two, a whole number of them, many; before, between and behind sequences of one row, two and none
    "many": [1] * 200 + [0] * 20 + [70, 128, 0, 64, 65] + [3000] + [2] * 100 + [63, 200],
    # the same among fewer than are numbered by their place
    "few": [1] * 100 + [0] * 20 + [70, 128, 0, 64, 65] + [3000] + [2] * 50 + [63, 200],
}


@pytest.mark.parametrize("which", LENS)
@pytest.mark.parametrize("dim,groups,states,dtype", [(64, 1, 16, F32), (70, 2, 5, F32), (40, 1, 40, F32), (70, 1, 16, BF16)])
def test_scan(lib, which, dim, groups, states, dtype):
    v, off, dev_off, dy, ds1 = scan.inputs(LENS[which], dim, groups, states, dtype, seed=len(LENS[which]) + states)
    f = scan.double(v)
    y, end = scan.forward(lib, v, dev_off)
    want, w_end = scan.reference(f, off, True)
    scan.close(y, want, scan.TOL[dtype], "y", scan.reference(scan.magnitudes(f), off, True)[0])
    scan.close(end, w_end, scan.TOL[F32], "end")
    got, g_want = scan.backward(lib, v, dev_off, dy, ds1), scan.wanted(v, off, dy, ds1, True)
    terms = scan.wanted(scan.magnitudes(v), off, dy.abs(), ds1.abs(), True)
    for k in scan.NAMES:
        scan.close(got[k], g_want[k], scan.tolerance(v[k]), k, terms[k])
    # the long sequence's own, which the others must not hide
    at = int(np.argmax(LENS[which]))
    rows = slice(int(off[at]), int(off[at + 1]))
    for k in ("x", "dt", "B", "C", "z"):
        scan.close(got[k][rows], g_want[k][rows], scan.tolerance(v[k]), k, terms[k][rows])
    scan.close(got["s0"][at], g_want["s0"][at], scan.TOL[F32], "s0", terms["s0"][at])


@pytest.mark.parametrize("which", LENS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_convolution(lib, which, dtype):
    i = conv.inputs(LENS[which], 70, 4, dtype, seed=3)
    got = lib.nugpr_short_conv_backward(i["x"], i["w"], i["dev_off"], i["dy"], bias=i["b"], silu=True, initial_state=i["s0"],
                                        d_final_state=i["ds1"])
    want = conv.wanted(i, i["b"], True, i["s0"], i["ds1"])
    for x, w, name in zip(got, want, ("dx", "dw", "db", "ds")):
        conv.close(x, w, conv.TOL[dtype], name)
    y, end = lib.nugpr_short_conv_forward(i["x"], i["w"], i["dev_off"], bias=i["b"], silu=True, initial_state=i["s0"])
    w, w_end = conv.reference(conv.double(i["x"]), conv.double(i["w"]), conv.double(i["b"]), i["off"], True, conv.double(i["s0"]))
    conv.close(y, w, conv.TOL[dtype], "y")
    assert torch.equal(end.double().cpu(), w_end)


def test_gradients_of_rates_at_the_ends_of_their_range(lib):
    """A = 0 keeps everything, -infinity nothing: gradients of all that these do not make infinity times zero (dt, with dt_bias and A's own).
    (The states that keep everything are sums of 300 terms that nothing scales down: four times the roundings.)"""
    v, off, dev_off, dy, ds1 = scan.inputs([5, 300, 0, 37], 40, 1, 8, F32, seed=21)
    v["A"][:, 0], v["A"][:, 1], v["A"][:, 2] = 0.0, float("-inf"), -1e38
    got, want = scan.backward(lib, v, dev_off, dy, ds1), scan.wanted(v, off, dy, ds1, True)
    terms = scan.wanted(scan.magnitudes(v), off, dy.abs(), ds1.abs(), True)
    for k in ("x", "B", "C", "D", "z", "s0"):
        scan.close(got[k], want[k], 4 * scan.TOL[F32], k, terms[k])
