"""Dropout into a residual: the generator's known answers, values and gradients bit for bit, sizes, types, states on the GPU."""
import math

import pytest
import torch

from paper_2505_11157_b200 import layer, sna
from test_layer_host import philox

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]


def kept(n, p, seed, offset):
    words = philox(-(-n // 4), seed, offset).reshape(-1)[:n]
    return torch.from_numpy(words >= min(2 ** 32 - 1, round(p * 2 ** 32))).cuda()


def definition(x, p, mask, residual):
    """As the kernel rounds: the product and the sum in 32 bits, the result to its type."""
    y = torch.where(mask.reshape(x.shape), x.float() * torch.tensor(1 / (1 - p), dtype=torch.float64).float().item(), 0.0)
    return (y if residual is None else y + residual.float()).to(x.dtype)


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda d: str(d).split(".")[1])
@pytest.mark.parametrize("shape", [(1,), (3,), (4, 1), (5, 7, 11), (4095,), (4096,), (2, 8192), (3, 91 * 181, 7)], ids=str)
@pytest.mark.parametrize("p", [0.0, 0.1, 0.75])
@pytest.mark.parametrize("with_residual", [False, True])
def test_values_and_gradients(shape, dtype, p, with_residual):
    torch.manual_seed(len(shape))
    x = torch.randn(shape, device="cuda").to(dtype).requires_grad_()
    residual = torch.randn(shape, device="cuda").to(dtype).requires_grad_() if with_residual else None
    seed, offset = -7 * 10 ** 17, 2 ** 63 - 1
    state = torch.tensor([seed, offset], device="cuda")
    out = layer.residual_dropout(x, state, p, residual)
    mask = kept(x.numel(), p, seed, offset)
    # one rounding differs where the compiler fuses the product and the sum: at most half a step of the product in 32 bits, then the type's
    ref = definition(x.detach(), p, mask, None if residual is None else residual.detach())
    if residual is None:
        assert torch.equal(out, ref)
    else:
        off = (out.double() - ref.double()).abs()
        bound = ref.double().abs() * torch.finfo(dtype).eps + (x.detach().double() / (1 - p)).abs() * 2.0 ** -23 + 1e-45
        assert bool((off <= bound).all())
        assert torch.equal(out[~mask.reshape(shape)], residual.detach()[~mask.reshape(shape)])
    dout = torch.randn(shape, device="cuda").to(dtype)
    grads = torch.autograd.grad(out, (x,) if residual is None else (x, residual), dout)
    assert torch.equal(grads[0], definition(dout, p, mask, None))
    if residual is not None:
        assert torch.equal(grads[1], dout)


def test_views_that_start_anywhere():
    for dtype in DTYPES:
        x = torch.randn(70001, device="cuda").to(dtype)
        state = torch.tensor([5, 6], device="cuda")
        for first in range(1, 9):
            view = x[first:]
            assert torch.equal(layer.residual_dropout(view, state, 0.3, view), layer.residual_dropout(view.clone(), state, 0.3, view.clone()))
    y = torch.randn(6, 5, 8, device="cuda").permute(2, 0, 1)
    assert torch.equal(layer.residual_dropout(y, state, 0.3, y), layer.residual_dropout(y.contiguous(), state, 0.3, y.contiguous()))


def test_share_of_kept_values_and_independence_of_offsets():
    x = torch.ones(1 << 22, device="cuda")
    a = layer.residual_dropout(x, torch.tensor([1, 0], device="cuda"), 0.1) != 0
    b = layer.residual_dropout(x, torch.tensor([1, 1], device="cuda"), 0.1) != 0
    # five standard deviations of a binomial count
    n = x.numel()
    assert abs(int(a.sum()) - 0.9 * n) < 5 * math.sqrt(n * 0.09) and abs(int((a & b).sum()) - 0.81 * n) < 5 * math.sqrt(n * 0.81 * 0.19)


def test_dropped_values_may_be_infinite_or_nan():
    x = torch.full((4096,), math.nan, device="cuda", dtype=torch.bfloat16)
    x[::2] = math.inf
    state = torch.tensor([11, 12], device="cuda")
    mask = kept(4096, 0.5, 11, 12)
    out = layer.residual_dropout(x, state, 0.5, torch.ones_like(x))
    assert bool((out[~mask] == 1).all()) and not bool(torch.isfinite(out[mask]).any())


def test_a_graph_draws_anew_and_its_gradient_uses_the_same_numbers():
    x = torch.randn(33, 1000, device="cuda").requires_grad_()
    ones = torch.ones_like(x)

    def step():
        state = layer.dropout_state("cuda")
        out = layer.residual_dropout(x, state, 0.4)
        return out, torch.autograd.grad(out, x, ones)[0]

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, grad = step()
    seen = []
    for _ in range(2):
        graph.replay()
        assert torch.equal(out != 0, grad != 0)
        seen.append(out.clone())
    assert not torch.equal(seen[0], seen[1])
    torch.manual_seed(9)
    first = layer.dropout_state("cuda")
    torch.manual_seed(9)
    assert torch.equal(first, layer.dropout_state("cuda"))


def test_a_state_that_changes_before_the_backward_pass_is_noticed():
    x = torch.randn(64, device="cuda").requires_grad_()
    state = torch.tensor([1, 2], device="cuda")
    out = layer.residual_dropout(x, state, 0.4)
    state += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


def test_empty_and_refusals():
    state = torch.tensor([1, 2], device="cuda")
    x = torch.randn(4, 8, device="cuda")
    assert layer.residual_dropout(x[:0], state, 0.4).shape == (0, 8)
    for args, says in [((x, state, 1.0), "less than 1"), ((x, state, -0.1), "at least 0"), ((x, state, math.nan), "at least 0"), ((x, state.int(), 0.1), "int64"),
                       ((x, state[:1], 0.1), "shape"), ((x, state.cpu(), 0.1), "CUDA tensor"), ((x.cpu(), state, 0.1), "CUDA tensor"), ((x.double(), state, 0.1), "float32"),
                       ((x, state, 0.1, x[:2]), "residual has shape"), ((x, state, 0.1, x.half()), "type of x"), ((x, state, 0.1, x.cpu()), "CUDA tensor")]:
        with pytest.raises(ValueError, match=says):
            layer.residual_dropout(*args)
    with pytest.raises(ValueError, match="plain torch.Tensor"):
        layer.residual_dropout(x.as_subclass(type("Sub", (torch.Tensor,), {})), state, 0.1)
