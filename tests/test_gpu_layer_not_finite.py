"""16-bit attention: infinities and NaN in queries and gradients stay where the definition leaves them; a row without points has zeros and no gradient whatever its
query holds, and a point left out has no gradient."""
import math

import pytest
import torch

from paper_2505_11157_b200 import layer

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16]
# queries, points: few queries, keys split over blocks, tiles of 64 stacked rows, tcgen05 (one tile, pieces, points brought together)
SIZES = [(1, 20), (3, 20000), (40, 40), (200, 300), (33, 9000), (4500, 4000)]


def tensors(Nq, Nk, dtype, C=32):
    torch.manual_seed(Nq + Nk)
    B, Hq, Hk = 3, 8, 4
    q, g = (torch.randn(B, Hq, 1, Nq, C, device="cuda").to(dtype) for _ in range(2))
    k, v = (torch.randn(B, Hk, 1, Nk, C, device="cuda").to(dtype) for _ in range(2))
    w = torch.randn(B, Nk, device="cuda")
    w[1] = -math.inf                                        # a field without points
    w[2, torch.rand(Nk, device="cuda") < 0.3] = -math.inf   # one with some
    w[2, 0] = 0.0
    return q, k, v, w, g


def run(q, k, v, w, g):
    ends = [x.detach().requires_grad_() for x in (q, k, v)]
    out, lse = layer.weighted_attention(*ends, w, return_lse=True)
    return (out.detach(), lse, *torch.autograd.grad(out, ends, g))


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda d: str(d).split(".")[1])
@pytest.mark.parametrize("Nq, Nk", SIZES)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_rows_without_points_whatever_their_query_holds(Nq, Nk, bad, dtype):
    q, k, v, w, g = tensors(Nq, Nk, dtype)
    with torch.no_grad():
        ref = layer.weighted_attention(q, k, v, w, return_lse=True)
        q[1, 0, 0, 0, 3] = q[1, 5, 0, Nq // 2, 0] = q[1, 7, 0, Nq - 1] = bad
        out, lse = layer.weighted_attention(q, k, v, w, return_lse=True)
        assert not bool(out[1].any()) and bool((lse[1] == -math.inf).all())
        assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])
        # points that take part: the row is NaN, and no other
        q[2, 6, 0, Nq - 1, 3] = bad
        out, lse = layer.weighted_attention(q, k, v, w, return_lse=True)
        assert bool(out[2, 6, 0, Nq - 1].isnan().all())
        out[2, 6, 0, Nq - 1], lse[2, 6, 0, Nq - 1] = ref[0][2, 6, 0, Nq - 1], ref[1][2, 6, 0, Nq - 1]
        assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda d: str(d).split(".")[1])
@pytest.mark.parametrize("Nq, Nk", SIZES)
@pytest.mark.parametrize("which", ["query", "gradient", "both"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_points_left_out_have_no_gradient_whatever_queries_and_gradients_hold(Nq, Nk, bad, which, dtype):
    q, k, v, w, g = tensors(Nq, Nk, dtype)
    clean = run(q, k, v, w, g)
    for x in [q] * (which != "gradient") + [g] * (which != "query"):
        x[1, 0, 0, 0, 3] = x[1, 5, 0, Nq // 2, 0] = x[1, 7, 0, Nq - 1] = bad      # in the field without points
    for got, ref in zip(run(q, k, v, w, g), clean):
        assert torch.equal(got, ref)
    for x in [q] * (which != "gradient") + [g] * (which != "query"):
        x[2, 6, 0, Nq - 1, 3] = bad         # and in one with some: key head 3 of that field has no gradient that is a number, the others have theirs
    _, _, dq, dk, dv = run(q, k, v, w, g)
    gone = w[2] == -math.inf
    assert not bool(dk[2, :, 0, gone].any()) and not bool(dv[2, :, 0, gone].any())
    assert bool(dq[2, 6, 0, Nq - 1].isnan().any()) and bool((~dk[2, 3, 0, ~gone].isfinite()).any())
    for got, ref in zip((dk, dv), clean[3:]):
        assert torch.equal(got[:2], ref[:2]) and torch.equal(got[2, :3], ref[2, :3])
    assert torch.equal(dq[:2], clean[2][:2]) and torch.equal(dq[2, :6], clean[2][2, :6])


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda d: str(d).split(".")[1])
@pytest.mark.parametrize("Nq, Nk", [(5, 20), (40, 40), (200, 300), (33, 9000), (4500, 4000)])
@pytest.mark.parametrize("bad", [math.nan, -math.nan, math.inf])
def test_a_gradient_that_is_not_finite_leaves_the_other_rows_theirs(Nq, Nk, bad, dtype):
    """float16: ds is held times a power of two from the largest rows of dout and v, without which values of this size overflow."""
    q, k, v, w, g = tensors(Nq, Nk, dtype)
    v *= 8
    g *= 64
    g[0, 2, 0, 1] = g[2, 6, 0, Nq - 1] = 0
    clean = run(q, k, v, w, g)[2]
    assert bool(clean.isfinite().all())
    g[0, 2, 0, 1, 5] = g[2, 6, 0, Nq - 1] = bad
    dq = run(q, k, v, w, g)[2]
    assert bool((~dq[0, 2, 0, 1].isfinite()).any()) and bool((~dq[2, 6, 0, Nq - 1].isfinite()).any())
    dq[0, 2, 0, 1], dq[2, 6, 0, Nq - 1] = clean[0, 2, 0, 1], clean[2, 6, 0, Nq - 1]
    assert torch.equal(dq, clean)
