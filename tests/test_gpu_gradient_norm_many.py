"""Norm and clipping of gradients (GPU) where one launch, or one pass of its workgroups, does not hold them: against float64, with the tolerances
of test_gpu_gradient_norm.py."""
import pytest
import torch

from test_gpu_gradient_norm import HALF, norm_of

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def check(lib, grads, to):
    """Beyond the bound, then within it."""
    for part in (0.3, 2.0):
        before, want = [g.clone() for g in grads], norm_of(grads)
        out = None if to is None else [torch.empty(g.shape, dtype=to, device="cuda") for g in grads]
        assert abs(float(lib.nugpr_gradient_norm(grads)) - want) <= 2.0 ** -24 * want
        got = lib.nugpr_clip_gradients(grads, part * want, out=out)
        assert abs(float(got) - want) <= 2.0 ** -24 * want
        for g, b, o in zip(grads, before, grads if out is None else out):
            if out is not None:
                assert torch.equal(g, b)
            exact = b.double() * min(1.0, part)
            assert bool(((o.double() - exact).abs() <= HALF[o.dtype] * exact.abs() * (1 + 2.0 ** -20) + 1e-44).all())


def random(n, dtype, gen):
    return torch.randn(n, generator=gen, device="cuda").to(dtype)


@pytest.mark.parametrize("to", [None, F32, BF16], ids=str)
def test_more_chunks_than_workgroups(lib, to):
    """40 million values: workgroups go on to a second part of them."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    check(lib, [random(n, t, gen) for n, t in ((20000003, BF16), (77, F32), (20000001, BF16), (1000001, F32))], to)


@pytest.mark.parametrize("to", [None, F32, BF16], ids=str)
def test_launches_without_values(lib, to):
    """Empty tensors that fill a launch of their own, in front, amid and behind."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    empty = [torch.empty(0, dtype=BF16, device="cuda")] * 300
    check(lib, empty + [random(1001, F32, gen)] + empty + [random(40000, BF16, gen), random(3, F32, gen)] + empty, to)
    assert float(lib.nugpr_gradient_norm(empty)) == 0.0 and float(lib.nugpr_clip_gradients(empty, 1.0)) == 0.0


@pytest.mark.parametrize("to", [None, F32], ids=str)
def test_thousands_of_tensors(lib, to):
    gen = torch.Generator(device="cuda").manual_seed(3)
    check(lib, [random(1 + 37 * i % 200, (F32, BF16)[i % 2], gen) for i in range(8000)], to)


def test_outputs_in_the_same_order(lib):
    """A dimension of one value has no order: its stride says nothing, whatever the other tensors are."""
    turned = torch.randn(40, 30, device="cuda").t()
    column = torch.randn(5, device="cuda").as_strided((5, 1), (1, 5))
    out = [torch.empty_strided(turned.shape, turned.stride(), device="cuda"), torch.empty(5, 1, device="cuda")]
    assert column.stride() != out[1].stride()
    lib.nugpr_clip_gradients([turned, column], 1e30, out=out)
    assert torch.equal(out[0], turned) and torch.equal(out[1], column)
    cube = torch.randn(6, 1, 7, device="cuda").transpose(0, 2)             # (7, 1, 6), strides 1, 7, 7
    to = torch.empty_strided((7, 1, 6), (1, 99, 7), device="cuda")
    lib.nugpr_clip_gradients([cube], 1e30, out=[to])
    assert torch.equal(to, cube)
    for bad in (torch.empty(30, 40, device="cuda"), torch.empty(60, 40, device="cuda")[::2]):
        with pytest.raises(lib.NugprError, match="shapes and strides"):
            lib.nugpr_clip_gradients([turned, column], 1.0, out=[bad, out[1]])
