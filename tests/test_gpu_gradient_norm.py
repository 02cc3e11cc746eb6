"""Norm and clipping of gradients (GPU) against float64.

Tolerances: the norm's squares are summed in 64 bits and it is rounded to float32 once, 2^-24 at most.  A clipped value is a
product in 64 bits, rounded to float32 and, where its buffer is bfloat16, to that: 2^-24, or 2^-8 and 2^-24."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8 + 2.0 ** -24}

SIZES = [[1], [3, 0, 5], [16384], [16385, 1, 7], [8191, 64, 100000, 33, 2], [5] * 300, [70001] * 3 + [0] * 130 + [9]]


def tensors(sizes, dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)
    types = [F32, BF16] if dtype is None else [dtype]
    return [torch.randn(n, generator=gen).to(types[i % len(types)]).cuda() for i, n in enumerate(sizes)]


def norm_of(grads):
    return float(sum(g.double().square().sum() for g in grads).sqrt())


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{s[0]}")
@pytest.mark.parametrize("dtype", [F32, BF16, None])
def test_norm(lib, sizes, dtype):
    grads = tensors(sizes, dtype)
    before = [g.clone() for g in grads]
    got, want = lib.nugpr_gradient_norm(grads), norm_of(grads)
    assert got.dtype == F32 and got.shape == ()
    assert abs(float(got) - want) <= 2.0 ** -24 * want
    assert all(torch.equal(a, b) for a, b in zip(grads, before))


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{s[0]}")
@pytest.mark.parametrize("dtype", [F32, BF16, None])
@pytest.mark.parametrize("to", ["in place", F32, BF16], ids=str)
def test_clip(lib, sizes, dtype, to):
    for part in (0.3, 2.0):
        grads = tensors(sizes, dtype)
        before = [g.clone() for g in grads]
        want = norm_of(grads)
        out = None if to == "in place" else [torch.empty(g.shape, dtype=to, device="cuda") for g in grads]
        got = lib.nugpr_clip_gradients(grads, part * want, out=out)
        assert abs(float(got) - want) <= 2.0 ** -24 * want
        for g, b, o in zip(grads, before, grads if out is None else out):
            if out is not None:
                assert torch.equal(g, b)
            exact = b.double() * min(1.0, part)
            assert bool(((o.double() - exact).abs() <= HALF[o.dtype] * exact.abs() * (1 + 2.0 ** -20) + 1e-44).all())
            if part > 1 and o.dtype == b.dtype:
                assert torch.equal(o, b)


def test_orders_and_alignments(lib):
    """Transposed tensors, slices that begin at any value, tensors without dimensions; a tensor with gaps is refused."""
    base = torch.randn(40, 30, device="cuda")
    flat = torch.randn(1001, device="cuda").to(BF16)
    grads = [base.t(), flat[1:400], flat[401:], torch.randn(3, 4, 5, device="cuda").permute(2, 0, 1), torch.tensor(2.0, device="cuda")]
    before, want = [g.clone() for g in grads], norm_of(grads)
    kept = flat[[0, 400]].clone()
    assert abs(float(lib.nugpr_clip_gradients(grads, 0.5 * want)) - want) <= 2.0 ** -24 * want
    for g, b in zip(grads, before):
        assert bool(((g.double() - 0.5 * b.double()).abs() <= 1.01 * HALF[g.dtype] * b.double().abs()).all())
    assert torch.equal(flat[[0, 400]], kept)
    out = [torch.empty_strided(g.shape, g.stride(), device="cuda") for g in grads]
    lib.nugpr_clip_gradients(grads, 1e30, out=out)
    assert all(torch.equal(o, g.float()) for o, g in zip(out, grads))
    with pytest.raises(lib.NugprError, match="one run of memory"):
        lib.nugpr_gradient_norm([base[:, ::2]])
    with pytest.raises(lib.NugprError, match="one run of memory"):
        lib.nugpr_gradient_norm([base[:1].expand(3, 30)])
    with pytest.raises(lib.NugprError, match="shapes and strides"):
        lib.nugpr_clip_gradients([base.t()], 1.0, out=[torch.empty(30, 40, device="cuda")])


def test_tensors_that_share_memory(lib):
    flat = torch.randn(100, device="cuda")
    for grads, out in (([flat, flat], None), ([flat[:60], flat[59:]], None), ([flat[:50], flat[50:]], [flat[1:51], torch.empty(50, device="cuda")]),
                       ([flat], [flat.view(BF16)[:100]])):
        with pytest.raises(lib.NugprError, match="overlap"):
            lib.nugpr_clip_gradients(grads, 1.0, out=out)
    both = float(lib.nugpr_gradient_norm([flat, flat]))                # (reading is no harm: it counts twice)
    assert abs(both - 2.0 ** 0.5 * norm_of([flat])) <= 2.0 ** -23 * both
    want = 0.5 * flat.clone()
    lib.nugpr_clip_gradients([flat[:60], flat[60:]], 0.5 * norm_of([flat]), out=[flat[:60], flat[60:]])    # its own place
    assert float((flat - want).abs().max()) <= 2.0 ** -23 * float(want.abs().max())


def test_large_and_small_values(lib):
    """Squares beyond the range of float32 on either side."""
    for scale in (1e30, 1e-30):
        g = torch.randn(1000, device="cuda") * scale
        want = norm_of([g])
        assert abs(float(lib.nugpr_gradient_norm([g])) - want) <= 2.0 ** -24 * want
        b = g.clone()
        lib.nugpr_clip_gradients([g], 1e-20)
        exact = b.double() * min(1.0, 1e-20 / want)
        assert bool(((g.double() - exact).abs() <= 2.0 ** -23 * exact.abs()).all())


def test_norms_that_are_not_finite(lib):
    g = torch.randn(100, device="cuda")
    g[7] = float("inf")
    assert float(lib.nugpr_clip_gradients([g], 1.0)) == float("inf")
    assert bool(torch.isnan(g[7])) and float(g[:7].abs().max()) == 0.0
    g = torch.randn(100, device="cuda")
    g[7] = float("nan")
    assert bool(torch.isnan(lib.nugpr_clip_gradients([g], 1.0))) and bool(torch.isnan(g).all())
    g, b = torch.randn(100, device="cuda"), None
    b = g.clone()
    lib.nugpr_clip_gradients([g], float("inf"))
    assert torch.equal(g, b)
    lib.nugpr_clip_gradients([g], 0.0)
    assert float(g.abs().max()) == 0.0
    assert float(lib.nugpr_clip_gradients([g], 0.0)) == 0.0


def test_refusals(lib):
    g = torch.randn(10, device="cuda")
    for call in (lambda: lib.nugpr_clip_gradients([g], -1.0), lambda: lib.nugpr_clip_gradients([g], float("nan")),
                 lambda: lib.nugpr_clip_gradients([], 1.0), lambda: lib.nugpr_gradient_norm([]),
                 lambda: lib.nugpr_gradient_norm([g.cpu()]), lambda: lib.nugpr_gradient_norm([g, g.cpu()]),
                 lambda: lib.nugpr_gradient_norm([g.double()]), lambda: lib.nugpr_clip_gradients([g], 1.0, out=[]),
                 lambda: lib.nugpr_clip_gradients([g], 1.0, out=[torch.empty(9, device="cuda")]),
                 lambda: lib.nugpr_clip_gradients([g], 1.0, out=[torch.empty(10, device="cuda").half()]),
                 lambda: lib.nugpr_gradient_norm([g.clone().requires_grad_()])):
        with pytest.raises(lib.NugprError):
            call()


def test_the_same_twice(lib):
    """No sum depends on the order in which workgroups run."""
    grads = tensors([100003, 5, 70000], BF16, seed=3)
    first = lib.nugpr_gradient_norm(grads)
    for _ in range(5):
        assert torch.equal(lib.nugpr_gradient_norm(grads), first)


def test_written_tensors_say_so(lib):
    g = torch.randn(10, device="cuda")
    before = g._version
    lib.nugpr_clip_gradients([g], 1.0)
    assert g._version == before + 1
