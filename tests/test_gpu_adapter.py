"""Projection with low-rank adapters (GPU) against float64.

Tolerances, relative in the 2-norm.  float32: sums of up to 4096 products whose roundings (2^-24 each, independent) grow with
the square root: 64 of them.  bfloat16: the result is rounded once to 8 significant bits, by up to 2^-8 of
a value each; the low-rank part keeps 16 bits on its way, 2^-16 more."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
TOL = {F32: 64 * 2.0 ** -24, BF16: 2.0 ** -8 + 2.0 ** -16}


def reference(x, W, A, B, off, which, scale, dy=None):
    x, W, A, B = (t.double().cpu() for t in (x, W, A, B))
    y = x @ W.T
    dA, dB = torch.zeros_like(A), torch.zeros_like(B)
    dx = None if dy is None else dy.double().cpu() @ W
    for s, a in enumerate(which):
        if not 0 <= a < A.shape[0]:
            continue
        r = slice(int(off[s]), int(off[s + 1]))
        y[r] += scale * (x[r] @ A[a].T) @ B[a]
        if dy is not None:
            d = dy.double().cpu()[r]
            dx[r] += scale * (d @ B[a].T) @ A[a]
            dA[a] += scale * (d @ B[a].T).T @ x[r]
            dB[a] += scale * (x[r] @ A[a].T).T @ d
    return y if dy is None else (dx, dA, dB)


def inputs(lens, inp, out, rank, n_adapters, dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)

    def r(*shape, scale=1.0):
        return (torch.randn(*shape, generator=gen) * scale).to(dtype).cuda()

    n = sum(lens)
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    which = torch.randint(0, n_adapters, (len(lens),), generator=gen).tolist()
    return (r(n, inp), r(out, inp, scale=inp ** -0.5), r(n_adapters, rank, inp, scale=inp ** -0.5),
            r(n_adapters, rank, out, scale=rank ** -0.5), off, torch.from_numpy(off).cuda(), which,
            torch.tensor(which, dtype=torch.int32, device="cuda"), r(n, out))


def close(x, want, tol):
    assert x.shape == want.shape
    err = float((x.double().cpu() - want).norm())
    assert err <= tol * float(want.norm()) or err == 0.0, err / float(want.norm() + 1e-300)


ROWS = [[1], [1] * 7, [0, 5, 0, 11, 1], [16, 16, 1, 31], [65], [1] * 130, [100, 0, 37, 300, 64, 3], [700, 513]]
DIMS = [(64, 64, 16), (256, 128, 4), (7, 3, 1), (100, 33, 5), (512, 20, 40), (1000, 777, 128), (96, 2048, 17)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lens", ROWS, ids=lambda l: "rows%d" % sum(l))
@pytest.mark.parametrize("inp,out,rank", DIMS)
def test_forward_and_backward(lib, lens, inp, out, rank, dtype):
    x, W, A, B, off, dev_off, which, dev_which, dy = inputs(lens, inp, out, rank, 3, dtype, seed=inp + len(lens))
    close(lib.nugpr_adapter_forward(x, W, A, B, dev_off, adapter_of=dev_which, scale=1.5),
          reference(x, W, A, B, off, which, 1.5), TOL[dtype])
    got = lib.nugpr_adapter_backward(x, W, A, B, dev_off, dy, adapter_of=dev_which, scale=1.5)
    for g, w in zip(got, reference(x, W, A, B, off, which, 1.5, dy)):
        assert g.dtype == dtype
        close(g, w, TOL[dtype])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_product(lib, dtype):
    """Whole tiles of every kind; the reference in float64 on the GPU."""
    x, W, A, B, off, dev_off, which, dev_which, dy = inputs([900, 1300, 1, 2000], 1024, 2048, 16, 4, dtype, seed=1)
    x64, W64, A64, B64, dy64 = (t.double() for t in (x, W, A, B, dy))
    y, dx = x64 @ W64.T, dy64 @ W64
    dA, dB = torch.zeros_like(A64), torch.zeros_like(B64)
    for s, a in enumerate(which):
        r = slice(int(off[s]), int(off[s + 1]))
        low, up = x64[r] @ A64[a].T, dy64[r] @ B64[a].T
        y[r] += low @ B64[a]
        dx[r] += up @ A64[a]
        dA[a] += up.T @ x64[r]
        dB[a] += low.T @ dy64[r]
    close(lib.nugpr_adapter_forward(x, W, A, B, dev_off, adapter_of=dev_which), y.cpu(), TOL[dtype])
    got = lib.nugpr_adapter_backward(x, W, A, B, dev_off, dy, adapter_of=dev_which)
    for g, w in zip(got, (dx, dA, dB)):
        close(g, w.cpu(), TOL[dtype])


@pytest.mark.parametrize("n", [5700, 2900])
@pytest.mark.parametrize("inp,out", [(192, 2104), (2104, 192)])
def test_tiles_of_256(lib, inp, out, n):
    """Enough rows and columns for the widest tiles (of 256 and of 128 rows), with both ends inside a tile, in either orientation of
    W; some requests end inside a tile, one has no adapter, and rows before the first and behind the last have no request."""
    x, W, A, B, _, _, _, _, dy = inputs([n], inp, out, 40, 3, BF16, seed=11)
    off, which = np.array([3, 700, 700, 701, n // 2, n - 10]), [1, 0, 2, -1, 0]
    dev_off, dev_which = torch.from_numpy(off).cuda(), torch.tensor(which, dtype=torch.int32, device="cuda")
    x64, W64, A64, B64, dy64 = (t.double() for t in (x, W, A, B, dy))
    y, dx = x64 @ W64.T, dy64 @ W64
    for s, a in enumerate(which):
        r = slice(int(off[s]), int(off[s + 1]))
        if a >= 0:
            y[r] += (x64[r] @ A64[a].T) @ B64[a]
            dx[r] += (dy64[r] @ B64[a].T) @ A64[a]
    close(lib.nugpr_adapter_forward(x, W, A, B, dev_off, adapter_of=dev_which), y.cpu(), TOL[BF16])
    close(lib.nugpr_adapter_backward(x, W, A, B, dev_off, dy, adapter_of=dev_which)[0], dx.cpu(), TOL[BF16])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,inp,out,rank", [(300, 520, 515, 20), (700, 1000, 1008, 5), (700, 1001, 999, 40), (1500, 1100, 1090, 33),
                                            (17000, 24, 31, 40), (200, 1300, 40, 9)])
def test_tiles_between(lib, n, inp, out, rank, dtype):
    """From too few tiles for all compute units to more than enough, aligned and not."""
    x, W, A, B, _, _, _, _, dy = inputs([n], inp, out, rank, 3, dtype, seed=12)
    off, which = np.array([3, 70, 70, 71, n // 2, n - 10]), [1, 0, 2, -1, 0]
    dev_off, dev_which = torch.from_numpy(off).cuda(), torch.tensor(which, dtype=torch.int32, device="cuda")
    x64, W64, A64, B64, dy64 = (t.double() for t in (x, W, A, B, dy))
    y, dx, dA, dB = x64 @ W64.T, dy64 @ W64, torch.zeros_like(A64), torch.zeros_like(B64)
    for s, a in enumerate(which):
        r = slice(int(off[s]), int(off[s + 1]))
        if a >= 0:
            low, up = x64[r] @ A64[a].T, dy64[r] @ B64[a].T
            y[r] += low @ B64[a]
            dx[r] += up @ A64[a]
            dA[a] += up.T @ x64[r]
            dB[a] += low.T @ dy64[r]
    close(lib.nugpr_adapter_forward(x, W, A, B, dev_off, adapter_of=dev_which), y.cpu(), TOL[dtype])
    got = lib.nugpr_adapter_backward(x, W, A, B, dev_off, dy, adapter_of=dev_which)
    for g, w in zip(got, (dx, dA, dB)):
        close(g, w.cpu(), TOL[dtype])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("inp,out,rank", [(200, 136, 8), (131, 203, 40), (70, 1200, 3)])
def test_many_requests_in_a_tile(lib, inp, out, rank, dtype):
    """Requests of none to four rows, one in seven without an adapter, one adapter with a value that is not finite."""
    lens = [s * 3 % 5 for s in range(70)]
    x, W, A, B, off, dev_off, _, _, dy = inputs(lens, inp, out, rank, 5, dtype, seed=13)
    which = [-1 if s % 7 == 3 else s % 5 for s in range(70)]
    dev_which = torch.tensor(which, dtype=torch.int32, device="cuda")
    bad_A, bad_B = A.clone(), B.clone()
    bad_A[2, rank - 1, inp - 1], bad_B[2, 0, 1] = float("nan"), float("inf")
    hit = torch.zeros(x.shape[0], dtype=torch.bool)
    for s, a in enumerate(which):
        hit[off[s]:off[s + 1]] = a == 2
    for AA, BB, rows in ((A, B, slice(None)), (bad_A, bad_B, ~hit)):
        close(lib.nugpr_adapter_forward(x, W, AA, BB, dev_off, adapter_of=dev_which, scale=1.5)[rows],
              reference(x, W, A, B, off, which, 1.5)[rows], TOL[dtype])
        dx = lib.nugpr_adapter_backward(x, W, AA, BB, dev_off, dy, adapter_of=dev_which, scale=1.5)[0]
        close(dx[rows], reference(x, W, A, B, off, which, 1.5, dy)[0][rows], TOL[dtype])


def test_gradient_against_differences(lib):
    """y is linear in x and bilinear in A and B: central differences of the float64 reference are exact."""
    x, W, A, B, off, dev_off, which, dev_which, dy = inputs([9, 40, 3], 50, 30, 6, 2, F32, seed=3)
    got = lib.nugpr_adapter_backward(x, W, A, B, dev_off, dy, adapter_of=dev_which, scale=0.5)
    gen = torch.Generator().manual_seed(1)
    base = [t.double().cpu() for t in (x, A, B)]
    for k in range(3):
        d = torch.randn(base[k].shape, generator=gen, dtype=torch.float64)
        f = []
        for sign in (1.0, -1.0):
            at = [t + sign * d if j == k else t for j, t in enumerate(base)]
            f.append(float((reference(at[0], W, at[1], at[2], off, which, 0.5) * dy.double().cpu()).sum()))
        along = float((got[k].double().cpu() * d).sum())
        assert abs(along - (f[0] - f[1]) / 2) <= TOL[F32] * float(got[k].double().norm()) * float(d.norm())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [40, 300])
def test_strides_and_offsets_in_storage(lib, rows, dtype):
    x, W, A, B, off, dev_off, which, dev_which, dy = inputs([rows - 7, 7], 96, 64, 8, 2, dtype, seed=4)
    wide = torch.full((rows, 200), float("nan"), dtype=dtype, device="cuda")
    for first in (8, 1):                                        # on 16 bytes, and not
        xs = wide[:, first:first + 96]
        xs.copy_(x)
        dys = torch.full((rows, 131), float("nan"), dtype=dtype, device="cuda")[:, first:first + 64]
        dys.copy_(dy)
        close(lib.nugpr_adapter_forward(xs, W, A, B, dev_off, adapter_of=dev_which), reference(x, W, A, B, off, which, 1.0), TOL[dtype])
        for g, w in zip(lib.nugpr_adapter_backward(xs, W, A, B, dev_off, dys, adapter_of=dev_which),
                        reference(x, W, A, B, off, which, 1.0, dy)):
            close(g, w, TOL[dtype])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [20, 200])
def test_rows_without_an_adapter(lib, rows, dtype):
    """Rows that no request owns, and requests whose adapter does not exist, get the projection alone."""
    x, W, A, B, _, _, _, _, dy = inputs([rows], 64, 48, 4, 2, dtype, seed=5)
    off = np.array([3, 9, 9, 15, rows - 1])
    which = [1, 0, -1, 2]
    dev = torch.from_numpy(off).cuda()
    dev_which = torch.tensor(which, dtype=torch.int32, device="cuda")
    close(lib.nugpr_adapter_forward(x, W, A, B, dev, adapter_of=dev_which), reference(x, W, A, B, off, which, 1.0), TOL[dtype])
    got = lib.nugpr_adapter_backward(x, W, A, B, dev, dy, adapter_of=dev_which)
    for g, w in zip(got, reference(x, W, A, B, off, which, 1.0, dy)):
        close(g, w, TOL[dtype])
    assert not got[1][0].any() and not got[2][0].any()          # the adapter of an empty request
    # offsets beyond the rows are taken as their ends; no adapters at all
    close(lib.nugpr_adapter_forward(x, W, A, B, torch.tensor([-4, 10, 10 ** 12], device="cuda")),
          reference(x, W, A, B, [0, 10, rows], [0, 1], 1.0), TOL[dtype])
    close(lib.nugpr_adapter_forward(x, W, A[:0], B[:0], dev), reference(x, W, A, B, off, [-1] * 4, 1.0), TOL[dtype])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [30, 400])
def test_values_that_are_not_finite_stay_with_their_rows(lib, rows, dtype):
    """One row of x and another request's adapter: only that row and that request's rows see them."""
    x, W, A, B, _, _, _, _, dy = inputs([rows], 64, 80, 4, 3, dtype, seed=6)
    off = np.array([0, 5, 14, rows])
    dev = torch.from_numpy(off).cuda()
    clean = reference(x, W, A, B, off, [0, 1, 2], 1.0)
    x2, A2, B2 = x.clone(), A.clone(), B.clone()
    x2[2, 7] = float("nan")
    A2[1, 0, 0] = float("inf")
    B2[1, 3, 5] = float("nan")
    y = lib.nugpr_adapter_forward(x2, W, A2, B2, dev).double().cpu()
    assert not torch.isfinite(y[2]).any() and not torch.isfinite(y[5:14]).any()
    keep = torch.ones(rows, dtype=torch.bool)
    keep[2] = False
    keep[5:14] = False
    close(y[keep], clean[keep], TOL[dtype])
    dx, dA, dB = lib.nugpr_adapter_backward(x2, W, A, B, dev, dy)
    want = reference(x, W, A, B, off, [0, 1, 2], 1.0, dy)
    close(dx, want[0], TOL[dtype])                               # (x is not in it)
    for g, w in ((dA, want[1]), (dB, want[2])):
        assert not torch.isfinite(g[0]).all()
        close(g[1:], w[1:], TOL[dtype])


def test_many_requests(lib):
    """More requests than a wave has lanes, several hundred with one row each, on a stream of their own."""
    lens = [1] * 300 + [0] * 70 + [2, 50] * 40
    x, W, A, B, off, dev_off, which, dev_which, dy = inputs(lens, 72, 40, 8, 20, F32, seed=7)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = lib.nugpr_adapter_forward(x, W, A, B, dev_off, adapter_of=dev_which)
        got = lib.nugpr_adapter_backward(x, W, A, B, dev_off, dy, adapter_of=dev_which)
    torch.cuda.current_stream().wait_stream(side)
    close(y, reference(x, W, A, B, off, which, 1.0), TOL[F32])
    for g, w in zip(got, reference(x, W, A, B, off, which, 1.0, dy)):
        close(g, w, TOL[F32])


def test_same_bits_again_and_in_a_graph(lib):
    x, W, A, B, off, dev_off, which, dev_which, dy = inputs([300, 5, 700], 256, 192, 16, 3, BF16, seed=8)

    def all_of_it():
        return (lib.nugpr_adapter_forward(x, W, A, B, dev_off, adapter_of=dev_which),
                *lib.nugpr_adapter_backward(x, W, A, B, dev_off, dy, adapter_of=dev_which))

    all_of_it()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_of_it()
    for _ in range(3):
        x.copy_(torch.randn(x.shape, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, all_of_it()):
            assert torch.equal(a, b)


def test_no_rows(lib):
    x, W, A, B, off, dev_off, which, dev_which, dy = inputs([0, 0], 64, 48, 4, 2, F32)
    assert lib.nugpr_adapter_forward(x, W, A, B, dev_off).shape == (0, 48)
    dx, dA, dB = lib.nugpr_adapter_backward(x, W, A, B, dev_off, dy)
    assert dx.shape == (0, 64) and not dA.any() and not dB.any()


def test_refusals(lib):
    x, W, A, B, off, dev_off, which, dev_which, dy = inputs([6, 2], 16, 12, 3, 2, F32)
    f = lib.nugpr_adapter_forward
    bad = [
        lambda: f(x.half(), W.half(), A.half(), B.half(), dev_off),
        lambda: f(x, W.to(BF16), A, B, dev_off),
        lambda: f(x[:, :15], W, A, B, dev_off),
        lambda: f(x, W.T.contiguous().T, A, B, dev_off),
        lambda: f(x, W, A[:1], B, dev_off),
        lambda: f(x, W, A, B[:, :2], dev_off),
        lambda: f(x, W, A, B, dev_off.int()),
        lambda: f(x, W, A, B, dev_off.cpu()),
        lambda: f(x, W, A, B, dev_off, adapter_of=dev_which[:1]),
        lambda: f(x, W, A, B, dev_off, adapter_of=dev_which.long()),
        lambda: f(x, W, A, B, dev_off, scale=float("inf")),
        lambda: f(x.T.contiguous().T, W, A, B, dev_off),
        lambda: f(x, W, torch.zeros(2, 129, 16, device="cuda"), torch.zeros(2, 129, 12, device="cuda"), dev_off),
        lambda: lib.nugpr_adapter_backward(x, W, A, B, dev_off, dy[:7]),
    ]
    for g in bad:
        with pytest.raises(lib.NugprError):
            g()
