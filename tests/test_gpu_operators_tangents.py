"""Inputs with a tangent (forward-mode derivatives): the operators say that they do not carry it on."""
import warnings

import pytest
import torch
import torch.autograd.forward_ad as forward_ad

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2207_09682_b200 import binding
    c = binding.Context(binding.make_params())
    yield c
    c.close()


def calls(ctx):
    """(name of the argument, a call of the tensor in its place, the tensor)."""
    f = lambda *s: torch.randn(s, device="cuda")  # noqa: E731
    x, g, w, b = f(4, 8), f(4, 8), f(8), f(8)
    r = ctx.layer_norm(x, w, b)
    states = lambda: [[torch.zeros(8, device="cuda")] for _ in range(2)]  # noqa: E731
    tokens, labels = torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    h, classes = f(4, 8).bfloat16(), f(3, 8).bfloat16()
    return [
        ("x", lambda t: ctx.layer_norm(t, w, b), x), ("weight", lambda t: ctx.layer_norm(x, t, b), w), ("bias", lambda t: ctx.layer_norm(x, w, t), b),
        ("grad_out", lambda t: ctx.layer_norm_backward(t, x, r.mean, r.rstd, w), g), ("x", lambda t: ctx.layer_norm_backward(g, t, r.mean, r.rstd, w), x),
        ("weight", lambda t: ctx.layer_norm_backward(g, x, r.mean, r.rstd, t), w), ("grads", lambda t: ctx.adamw([b.clone()], [t], *states(), 1, 0.1), w),
        ("table", lambda t: ctx.embed(t, tokens), x), ("hidden", lambda t: ctx.softmax_ce(t, classes, labels), h), ("gradients", lambda t: ctx.clip_grad_norm([t], float("inf")), g),
    ]


def test_a_tangent_is_not_lost_without_a_word(ctx):
    for name, call, t in calls(ctx):
        with warnings.catch_warnings():
            warnings.simplefilter("error")
            call(t)
        with forward_ad.dual_level():
            dual = forward_ad.make_dual(t, torch.ones_like(t))
            with pytest.warns(UserWarning, match="%s has a tangent" % name):
                call(dual)
            with warnings.catch_warnings():
                warnings.simplefilter("error")
                call(forward_ad.unpack_dual(dual).primal)
                with pytest.raises(UserWarning):
                    call(dual)


def test_a_gradient_and_a_tangent(ctx):
    """Both are told; without gradients the tangent alone, which torch.no_grad() does not silence."""
    x = torch.randn((4, 8), device="cuda", requires_grad=True)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, torch.ones_like(x))
        with pytest.warns(UserWarning) as told:
            ctx.layer_norm(dual)
        assert ["requires a gradient" in str(t.message) for t in told] == [True, False]
        with torch.no_grad(), pytest.warns(UserWarning) as told:
            ctx.layer_norm(dual)
        assert len(told) == 1 and "has a tangent" in str(told[0].message)
