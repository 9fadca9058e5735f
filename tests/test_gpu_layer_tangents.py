"""Forward-mode differentiation: the layer's operators have no rule for it, so a tensor with a tangent is refused; nothing comes back as a derivative of zero."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad

from paper_2505_11157_b200 import layer

pytestmark = pytest.mark.gpu


def inputs():
    torch.manual_seed(0)
    q, k, v = (torch.randn(1, 2, 3, 4, 16, device="cuda").half() for _ in range(3))
    w, log_weights = torch.ones(16, device="cuda"), torch.zeros(12, device="cuda")
    rotation = layer.rotation_tables(3, 4, [[0.1], [0.2], [0.3]], [1])
    return q, k, v, w, log_weights, rotation, layer.dropout_state("cuda")


CALLS = {
    "q, norm": lambda d, q, k, v, w, lw, r, s: layer.qk_norm_rotate(d(q), k),
    "k, norm": lambda d, q, k, v, w, lw, r, s: layer.qk_norm_rotate(q, d(k)),
    "q_weight": lambda d, q, k, v, w, lw, r, s: layer.qk_norm_rotate(q, k, d(w)),
    "k_weight": lambda d, q, k, v, w, lw, r, s: layer.qk_norm_rotate(q, k, None, d(w)),
    "table": lambda d, q, k, v, w, lw, r, s: layer.qk_norm_rotate(q, k, None, None, None, (r[0], d(r[1]))),
    "q, attention": lambda d, q, k, v, w, lw, r, s: layer.weighted_attention(d(q), k, v),
    "k, attention": lambda d, q, k, v, w, lw, r, s: layer.weighted_attention(q, d(k), v),
    "v, attention": lambda d, q, k, v, w, lw, r, s: layer.weighted_attention(q, k, d(v)),
    "log_weights": lambda d, q, k, v, w, lw, r, s: layer.weighted_attention(q, k, v, d(lw)),
    "x": lambda d, q, k, v, w, lw, r, s: layer.residual_dropout(d(q), s, 0.5),
    "residual": lambda d, q, k, v, w, lw, r, s: layer.residual_dropout(q, s, 0.5, d(k)),
}


@pytest.mark.parametrize("requires_grad", [False, True])
@pytest.mark.parametrize("name", CALLS)
def test_an_argument_with_a_tangent_is_refused(name, requires_grad):
    args = inputs()
    with forward_ad.dual_level():
        dual = lambda t: forward_ad.make_dual(t.clone().requires_grad_() if requires_grad and name not in ("table", "log_weights") else t, torch.ones_like(t))
        with pytest.raises(RuntimeError, match="tangent"):
            CALLS[name](dual, *args)
        CALLS[name](lambda t: t, *args)


@pytest.mark.parametrize("call", [lambda x, s: layer.qk_norm_rotate(x, x)[0], lambda x, s: layer.weighted_attention(x, x, x), lambda x, s: layer.residual_dropout(x, s, 0.5),
                                  lambda x, s: layer.residual_dropout(x.detach(), s, 0.5, x)], ids=["norm", "attention", "dropout", "residual"])
def test_a_gradient_with_a_tangent_is_refused(call):
    x, *_, state = inputs()
    x.requires_grad_()
    with forward_ad.dual_level():
        y = call(x, state)
        g = torch.ones_like(y)
        with pytest.raises(RuntimeError, match="tangent"):
            torch.autograd.grad(y, x, forward_ad.make_dual(g, g), retain_graph=True)
        assert bool(torch.isfinite(torch.autograd.grad(y, x, g)[0]).all())


def test_without_forward_mode_the_value_alone_counts():
    q, k, v, *_ = inputs()
    ref = layer.weighted_attention(q, k, v)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(q, torch.ones_like(q))
        with torch.inference_mode():
            assert torch.equal(layer.weighted_attention(dual, k, v), ref)
