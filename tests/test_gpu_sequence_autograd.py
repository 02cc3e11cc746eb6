"""The sequence operators (GPU) and autograd, which does not record them: no gradient is lost in silence."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def attention():
    gen = torch.Generator().manual_seed(0)

    def r(*shape):
        return torch.randn(*shape, generator=gen).cuda()

    return dict(q=r(9, 2, 16), k=r(9, 2, 16), v=r(9, 2, 8), log_decay=-r(2).abs(), seq_offsets=torch.tensor([0, 4, 9], device="cuda")), \
        r(9, 2, 8), r(2, 2, 16, 8)


def adapters():
    gen = torch.Generator().manual_seed(1)

    def r(*shape):
        return torch.randn(*shape, generator=gen).cuda()

    return dict(x=r(9, 16), W=r(12, 16), A=r(2, 3, 16), B=r(2, 3, 12), seq_offsets=torch.tensor([0, 4, 9], device="cuda")), r(9, 12)


def calls(lib):
    a, d_o, state = attention()
    yield lib.nugpr_decay_attention_forward, dict(a, initial_state=state), ("q", "k", "v", "log_decay", "initial_state")
    yield lib.nugpr_decay_attention_backward, dict(a, d_o=d_o, initial_state=state, d_final_state=state), ("q", "k", "v", "log_decay", "d_o", "initial_state", "d_final_state")
    one = {name: t[:2] if name in "qkv" else t for name, t in a.items() if name != "seq_offsets"}
    yield lib.nugpr_decay_attention_step, dict(one, state=state), ("q", "k", "v", "log_decay", "state")
    p, d_y = adapters()
    yield lib.nugpr_adapter_forward, p, ("x", "W", "A", "B")
    yield lib.nugpr_adapter_backward, dict(p, d_y=d_y), ("x", "W", "A", "B", "d_y")


def test_inputs_that_require_gradients_are_refused(lib):
    for call, args, names in calls(lib):
        for name in names:
            given = dict(args, **{name: args[name].detach().clone().requires_grad_()})
            with pytest.raises(lib.NugprError, match=name):
                call(**given)
            with torch.no_grad():
                call(**given)


def test_the_calls_serve_an_autograd_function(lib):
    class Project(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, W, A, B, offsets):
            ctx.save_for_backward(x, W, A, B, offsets)
            return lib.nugpr_adapter_forward(x, W, A, B, offsets)

        @staticmethod
        def backward(ctx, d_y):
            dx, dA, dB = lib.nugpr_adapter_backward(*ctx.saved_tensors, d_y.contiguous())
            return dx, None, dA, dB, None

    p, d_y = adapters()
    x, A, B = (p[n].requires_grad_() for n in ("x", "A", "B"))
    Project.apply(x, p["W"], A, B, p["seq_offsets"]).backward(d_y)
    with torch.no_grad():
        want = lib.nugpr_adapter_backward(x, p["W"], A, B, p["seq_offsets"], d_y)
    for got, w in zip((x.grad, A.grad, B.grad), want):
        assert torch.equal(got, w)


def test_a_step_says_that_it_has_written_the_state(lib):
    a, _, state = attention()
    del a["seq_offsets"]
    one = {name: t[:2] if name in "qkv" else t for name, t in a.items()}
    weight = torch.randn(state.shape, device="cuda", requires_grad=True)
    y = (weight * state).sum()                       # keeps the state for the gradient of weight
    before = state._version
    lib.nugpr_decay_attention_step(**one, state=state)
    assert state._version == before + 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    with torch.inference_mode():
        lib.nugpr_decay_attention_step(**one, state=state.clone())
