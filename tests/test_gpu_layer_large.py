"""The layer's operators on tensors of more than 2^31 (dropout: 2^34) elements: offsets beyond 32 bits."""
import math

import pytest
import torch

from paper_2505_11157_b200 import layer
from test_layer_host import philox

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("Nq", [2, 40])
def test_attention_over_a_long_field(Nq):
    """Only the first and the last points take part, and in one more field points beyond 2^31 elements: as over those alone."""
    torch.manual_seed(Nq)
    C, Nk, ends = 128, (1 << 24) + 333, 500
    q, g = (torch.randn(2, 2, 1, Nq, C, device="cuda").bfloat16() for _ in range(2))
    k, v = (torch.zeros(2, 1, 1, Nk, C, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    w = torch.full((Nk,), -math.inf, device="cuda")
    index = torch.cat((torch.arange(ends), torch.arange(Nk - ends, Nk))).cuda()
    small = [torch.randn(2, 1, 1, 2 * ends, C, device="cuda").bfloat16() for _ in range(2)]
    for x, y in zip((k, v), small):
        x.index_copy_(3, index, y)
    w[index] = torch.randn(2 * ends, device="cuda")

    def run(k, v, w):
        ends = [x.detach().requires_grad_() for x in (q, k, v)]
        out = layer.weighted_attention(*ends, w)
        return (out.detach(), *torch.autograd.grad(out, ends, g))

    out, dq, dk, dv = run(k, v, w)
    ref = run(*small, w[index])
    off = lambda a, b: float((a.double() - b.double()).norm() / b.double().norm())
    # (both are off by up to a step of bfloat16 in norm from the definition)
    for got, right in ((out, ref[0]), (dq, ref[1]), (dk.index_select(3, index), ref[2]), (dv.index_select(3, index), ref[3])):
        assert off(got, right) < 2 * torch.finfo(torch.bfloat16).eps
    assert not any(bool(x[:, :, :, ends:ends + 10 ** 6].any()) or bool(x[:, :, :, Nk - ends - 10 ** 6:Nk - ends].any()) for x in (dk, dv))


def test_norm_and_rotation_of_a_large_tensor():
    torch.manual_seed(1)
    B, H, grid, C = 2, 16, (1024, 1025), 64         # (2.1e9 elements)
    x = torch.randn(1, 1, *grid, C, device="cuda", dtype=torch.bfloat16)
    big = x.repeat(B, H, 1, 1, 1).requires_grad_()
    w = torch.rand(C, device="cuda")
    rotation = layer.rotation_tables(*grid, torch.rand(grid[0], 16), list(range(16)))
    with torch.no_grad():
        ref = layer.qk_norm_rotate(x, x, w, w, rotation, rotation)[0]
    y = layer.qk_norm_rotate(big, big.detach()[:, :1], w, w, rotation, rotation)[0]
    assert all(torch.equal(y[b, h], ref[0, 0]) for b in range(B) for h in (0, 7, 15))
    xr = x.clone().requires_grad_()
    want = torch.autograd.grad(layer.qk_norm_rotate(xr, x, w, w, rotation, rotation)[0], xr, x)[0]
    got = torch.autograd.grad(y, big, big.detach())[0]
    assert all(torch.equal(got[b, h], want[0, 0]) for b in range(B) for h in (0, 7, 15))


def test_dropout_of_many_values():
    n, p, seed, offset = (1 << 34) + 4099, 0.3, 123456789, 42        # (the counter's second word is one behind 2^34)
    x = torch.ones(n, device="cuda", dtype=torch.bfloat16)
    out = layer.residual_dropout(x, torch.tensor([seed, offset], device="cuda"), p)
    kept = torch.tensor(1 / (1 - p)).bfloat16().item()
    for first in (0, (1 << 32) - 2048, (1 << 34) - 2048):
        words = philox(1024 + (256 if first == 0 else 0), seed, offset, first=first // 4).reshape(-1)
        mask = torch.from_numpy(words >= round(p * 2 ** 32)).cuda()
        assert torch.equal(out[first:first + mask.numel()].float(), torch.where(mask, kept, 0.0))
    words = philox(2, seed, offset, first=n // 4).reshape(-1)[:n % 4]
    assert torch.equal(out[n - n % 4:].float().cpu(), torch.where(torch.from_numpy(words >= round(p * 2 ** 32)), kept, 0.0))
