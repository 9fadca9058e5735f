"""16-bit attention: errors of whole results, in their 2-norm.

The bounds per element (test_gpu_layer_attention.py) add up every rounding in its worst direction, which over thousands of points leaves room for a lost block.  A
2-norm does not: results of random data are sums of terms of random signs, each off by its own roundings.  With u half a step, the result's own rounding (at most u,
root mean square u / sqrt 3) and those of p and ds, the operands of the second products (the same of each term), give sqrt(3) u / sqrt(3) = u if none is averaged
out; sums in 32 bits and exponentials (2^-18.5) are far below.  Twice that is allowed, and the test makes sure that it shows a lost block of 64 points."""
import math

import pytest
import torch

from paper_2505_11157_b200 import layer

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16]
# B, Hq, Hk, queries, points, C: one tile, pieces of the last wave, pieces of long walks on either side, two-part operands, wide heads, shared heads, mma.sync (few
# queries; few points), points brought together
SHAPES = [(2, 4, 2, 200, 300, 32), (1, 4, 4, 2048, 2048, 32), (1, 1, 1, 33, 9800, 32), (2, 4, 1, 17, 20011, 64), (1, 2, 2, 20011, 65, 40), (1, 4, 1, 9001, 130, 128),
          (2, 4, 2, 800, 1203, 8), (1, 8, 8, 4000, 1500, 128), (2, 3, 3, 129, 5000, 96), (2, 8, 2, 1, 30011, 64), (2, 8, 2, 16, 4099, 64), (1, 4, 2, 3000, 61, 24),
          (3, 8, 2, 5500, 1030, 40), (2, 4, 4, 4100, 4200, 128)]


def definition(q, k, v, w, g):
    """out, dq, dk, dv in 64 bits, and of each the 2-norm of what one block of 64 points (dk, dv: of 64 queries of one head) contributes."""
    B, Hq, Hk, C = q.shape[0], q.shape[1], k.shape[1], q.shape[-1]
    Q, Y, K, V = (x.double().reshape(B, Hk, -1, C) for x in (q, g, k, v))
    gone = (w == -math.inf).reshape(-1, 1, w.shape[-1], 1)
    K, V = K.masked_fill(gone, 0.0), V.masked_fill(gone, 0.0)
    s = Q @ K.transpose(2, 3) * C ** -0.5 + w.double()[:, None, None, :]
    p = torch.softmax(s, -1)
    out = p @ V
    ds = p * (Y @ V.transpose(2, 3) - (Y * out).sum(-1, keepdim=True))
    values = [out, C ** -0.5 * ds @ K, C ** -0.5 * ds.transpose(2, 3) @ Q, p.transpose(2, 3) @ Y]
    points = torch.nonzero(~(w == -math.inf).any(0)).flatten()[:64]       # (a block's worth of points that take part)
    rows = slice(0, min(64, q.shape[3]))
    lost = [p[..., points] @ V[:, :, points], C ** -0.5 * ds[..., points] @ K[:, :, points], C ** -0.5 * ds[:, :, rows].transpose(2, 3) @ Q[:, :, rows],
            p[:, :, rows].transpose(2, 3) @ Y[:, :, rows]]
    return [x.reshape(y.shape) for x, y in zip(values, (q, q, k, v))], [float(x.norm()) for x in lost]


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda d: str(d).split(".")[1])
@pytest.mark.parametrize("share", [0.0, 0.3])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_errors_of_whole_results(shape, share, dtype):
    B, Hq, Hk, Nq, Nk, C = shape
    torch.manual_seed(Nq + Nk)
    q, g = (torch.randn(B, Hq, 1, Nq, C, device="cuda").to(dtype) for _ in range(2))
    k, v = (torch.randn(B, Hk, 1, Nk, C, device="cuda").to(dtype) for _ in range(2))
    w = torch.randn(B, Nk, device="cuda").masked_fill(torch.rand(B, Nk, device="cuda") < share, -math.inf)
    ends = [x.requires_grad_() for x in (q, k, v)]
    out = layer.weighted_attention(*ends, w)
    got = [out.detach(), *torch.autograd.grad(out, ends, g)]
    with torch.no_grad():
        values, lost = definition(q, k, v, w, g)
    bound = torch.finfo(dtype).eps
    for name, x, ref, block in zip(("out", "dq", "dk", "dv"), got, values, lost):
        size = float(ref.norm())
        assert block > 4 * bound * size, (name, block / size)
        assert float((x.double() - ref).norm()) <= bound * size, (name, float((x.double() - ref).norm()) / size)


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda d: str(d).split(".")[1])
@pytest.mark.parametrize("shape", [(2, 8, 2, 1, 361 * 720, 64), (1, 2, 2, 1, 30011, 128), (2, 8, 1, 2, 9000, 32), (4, 8, 2, 2, 16200, 40), (1, 4, 4, 16, 8192, 32), (2, 4, 2, 60, 50, 24)],
                         ids=lambda s: "-".join(map(str, s)))
def test_few_queries_or_points_are_off_by_the_rounding_of_the_result_alone(shape, dtype):
    """p in two 16-bit parts is off by u^2, exponentials by 2^-22, sums in 32 bits by less than a thousandth of u on average; an error d before the result's rounding moves
    the result by at most 2 d more than that rounding, so that a twentieth of it is ample."""
    B, Hq, Hk, Nq, Nk, C = shape
    torch.manual_seed(Nk)
    q, k, v = (torch.randn(B, h, 1, n, C, device="cuda").to(dtype) for h, n in ((Hq, Nq), (Hk, Nk), (Hk, Nk)))
    w = torch.randn(B, Nk, device="cuda")
    ref = definition(q, k, v, w, torch.zeros_like(q))[0][0]
    alone = float((ref.to(dtype).double() - ref).norm())
    assert float((layer.weighted_attention(q, k, v, w).double() - ref).norm()) < 1.05 * alone
