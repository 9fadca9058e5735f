"""Norm and rotation of queries and keys against their definition in 64 bits: types, head widths, strides, pairs, odd grids, gradients."""
import math

import pytest
import torch

from paper_2505_11157_b200 import layer, sna

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
U32 = 2.0 ** -24


def tables(nlat, nlon, pairs_lat, pairs_lon):
    lat_angles = torch.arange(nlat, dtype=torch.float64)[:, None] * (0.7 + torch.arange(pairs_lat, dtype=torch.float64))
    return layer.rotation_tables(nlat, nlon, lat_angles, [1 + 3 * p for p in range(pairs_lon)])


def definition(x, weight, rotation, eps, interleaved):
    """In 64 bits, and the size of the terms that each value is a sum of."""
    x = x.double()
    n = x / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    if weight is not None:
        n = n * weight.double()
    y, size = n.clone(), n.abs()
    if rotation is not None:
        lat, lon = (t.double() for t in rotation)
        pairs_lat, pairs = lat.shape[1], lat.shape[1] + lon.shape[1]
        y, size = [n[..., c] for c in range(n.shape[-1])], [n[..., c].abs() for c in range(n.shape[-1])]
        for p in range(pairs):
            a, b = (2 * p, 2 * p + 1) if interleaved else (p, p + pairs)
            cos, sin = (lat[:, None, p, 0], lat[:, None, p, 1]) if p < pairs_lat else (lon[None, :, p - pairs_lat, 0], lon[None, :, p - pairs_lat, 1])
            y[a], y[b] = n[..., a] * cos - n[..., b] * sin, n[..., a] * sin + n[..., b] * cos
            size[a] = size[b] = n[..., a].abs() + n[..., b].abs()
        y, size = torch.stack(y, -1), torch.stack(size, -1)
    return y, size


def near(got, ref, size, steps, dtype, what):
    """`steps` roundings to 32 bits of terms of that size, and the result's own to its type; 16-bit floats also end at a smallest number."""
    tol = steps * U32 * size + (torch.finfo(dtype).eps / 2) * ref.abs() + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    off = (got.double() - ref).abs()
    assert got.dtype == dtype and bool((off <= tol).all()), (what, float((off / tol).max()))


def heads(B, H, nlat, nlon, C, dtype, order="plain"):
    if order == "plain":
        return torch.randn(B, H, nlat, nlon, C, device="cuda").to(dtype)
    if order == "points first":
        return torch.randn(B, nlat, nlon, H, C, device="cuda").to(dtype).permute(0, 3, 1, 2, 4)
    if order == "packed":                 # a slice of a packed projection, with its neighbours around it
        return torch.randn(B, nlat, nlon, 3, H, C, device="cuda").to(dtype)[:, :, :, 1].permute(0, 3, 1, 2, 4)
    if order == "shared":                 # one head seen as H
        return torch.randn(B, 1, nlat, nlon, C, device="cuda").to(dtype).expand(B, H, nlat, nlon, C)
    if order == "odd":                    # rows that start where no load of 8 bytes may
        return torch.randn(B, H, nlat, nlon, C + 1, device="cuda").to(dtype)[..., 1:]
    if order == "channels apart":
        return torch.randn(B, H, C, nlat, nlon, device="cuda").to(dtype).permute(0, 1, 3, 4, 2)
    raise AssertionError(order)


CASES = [
    # B, Hq, Hk, q grid, k grid, C, pairs_lat, pairs_lon, interleaved, order
    (1, 1, 1, (1, 1), (1, 1), 4, 1, 1, False, "plain"),
    (2, 4, 4, (5, 9), (5, 9), 32, 8, 8, False, "plain"),
    (2, 4, 2, (7, 13), (14, 26), 64, 8, 8, True, "points first"),
    (3, 6, 2, (3, 67), (9, 5), 24, 5, 6, False, "packed"),
    (1, 5, 1, (33, 17), (2, 301), 128, 0, 64, False, "plain"),
    (1, 5, 1, (33, 17), (2, 301), 128, 32, 0, True, "shared"),
    (2, 3, 3, (4, 5), (1, 7), 20, 3, 4, False, "odd"),
    (2, 3, 3, (4, 5), (1, 7), 100, 1, 0, True, "channels apart"),
    (2, 2, 2, (6, 6), (6, 6), 12, 0, 0, False, "plain"),
    (9, 8, 8, (2, 3), (2, 3), 16, 4, 4, False, "plain"),
    (1, 2, 2, (90, 181), (180, 362), 8, 2, 2, False, "points first"),
]


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda d: str(d).split(".")[1])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_values_and_gradients(case, dtype):
    B, Hq, Hk, q_grid, k_grid, C, pairs_lat, pairs_lon, interleaved, order = case
    torch.manual_seed(C + B)
    q, k = heads(B, Hq, *q_grid, C, dtype, order).detach().requires_grad_(), heads(B, Hk, *k_grid, C, dtype, order).detach().requires_grad_()
    weights = [torch.randn(C, device="cuda").requires_grad_() for _ in range(2)]
    rotations = [tables(*q_grid, pairs_lat, pairs_lon), tables(*k_grid, pairs_lat, pairs_lon)]
    eps = 1e-3
    out = layer.qk_norm_rotate(q, k, *weights, *rotations, eps=eps, interleaved=interleaved)
    grads_out = [heads(*o.shape, dtype, "points first" if order == "plain" else "plain") for o in out]
    got = torch.autograd.grad(out, (q, k, *weights), grads_out, retain_graph=True)
    again = torch.autograd.grad(out, (q, k, *weights), grads_out)
    for i, (x, weight, rotation) in enumerate(zip((q, k), weights, rotations)):
        ends = [x.detach().double().requires_grad_(), weight.detach().double().requires_grad_()]
        ref, size = definition(*ends, rotation, eps, interleaved)
        # mean of C squares, its root, three products, one sum
        near(out[i].detach(), ref.detach(), size.detach(), C + 16, dtype, f"out {i}")
        g = grads_out[i].double()
        ref_x, ref_w = torch.autograd.grad(ref, ends, g)
        xd = x.detach().double()
        r = 1 / (xd.square().mean(-1, keepdim=True) + eps).sqrt()
        turned = definition_transposed_size(g, rotation, interleaved)
        gw = turned * weight.detach().double().abs()
        size_x = r * (gw + xd.abs() * r * (gw * xd.abs() * r).mean(-1, keepdim=True))
        near(got[i], ref_x, size_x, 3 * C + 32, dtype, f"dx {i}")
        rows = x.numel() // C
        near(got[2 + i], ref_w, (turned * xd.abs() * r).sum((0, 1, 2, 3)), C + 16 + rows, torch.float32, f"dw {i}")
        assert torch.equal(got[i], again[i]) and torch.equal(got[2 + i], again[2 + i])


def definition_transposed_size(g, rotation, interleaved):
    """Bound of |R^T g|: the two terms of each pair."""
    pairs = rotation[0].shape[1] + rotation[1].shape[1]
    size = g.abs().clone()
    for p in range(pairs):
        a, b = (2 * p, 2 * p + 1) if interleaved else (p, p + pairs)
        size[..., a] = size[..., b] = g[..., a].abs() + g[..., b].abs()
    return size


@pytest.mark.parametrize("B, H, grid, C, dtype", [(1, 3, (64, 128), 32, torch.float32), (1, 1, (91, 181), 8, torch.bfloat16), (3, 7, (45, 90), 64, torch.float16),
                                                  (5, 5, (7, 9), 128, torch.bfloat16), (1, 17, (30, 61), 16, torch.float32), (3, 1, (180, 361), 24, torch.float32)])
def test_gradients_of_the_weights_closely(B, H, grid, C, dtype):
    """Odd numbers of slices, several points per thread.  A sum passes a thread's vectors (at most 64 here), up to 256 threads of a block, and up to 10 + 7 partial
    sums: no more than 400 roundings to 32 bits, of which each is of a part of the sum of the terms' magnitudes."""
    torch.manual_seed(C)
    q, k = heads(B, H, *grid, C, dtype), heads(B, 1, *grid, C, dtype)
    weights = [torch.randn(C, device="cuda").requires_grad_() for _ in range(2)]
    rotation = tables(*grid, C // 4, C // 4)
    out = layer.qk_norm_rotate(q, k, *weights, rotation, rotation)
    grads_out = [torch.randn(o.shape, device="cuda").to(dtype) for o in out]
    got = torch.autograd.grad(out, weights, grads_out)
    for x, weight, g, dw in zip((q, k), weights, grads_out, got):
        w = weight.detach().double().requires_grad_()
        ref = torch.autograd.grad(definition(x, w, rotation, 1e-6, False)[0], w, g.double())[0]
        n = x.double().abs() / (x.double().square().mean(-1, keepdim=True) + 1e-6).sqrt()
        near(dw, ref, (definition_transposed_size(g.double(), rotation, False) * n).sum((0, 1, 2, 3)), C + 416, torch.float32, "dw")


def test_results_in_place_of_inputs():
    """Through the C ABI: y is x, and dx is dy."""
    torch.manual_seed(11)
    x, w = heads(2, 3, 5, 7, 24, torch.bfloat16), torch.randn(24, device="cuda")
    rotation = tables(5, 7, 5, 6)
    xr = x.clone().requires_grad_()
    y = layer.qk_norm_rotate(xr, xr.detach(), w, w, rotation, rotation, eps=0.5)[0]
    g = heads(2, 3, 5, 7, 24, torch.bfloat16)
    dx = torch.autograd.grad(y, xr, g)[0]
    t = lambda a: sna.SnaTensor(a.data_ptr(), a.stride(0), a.stride(1), a.stride(2), a.stride(3))
    stream = torch.cuda.current_stream().cuda_stream
    a, b = x.clone(), g.clone()
    part = sna.SnaRotate(nlat=5, nlon=7, H=3, x=t(a), y=t(a), weight=w.data_ptr(), lat_table=rotation[0].data_ptr(), lon_table=rotation[1].data_ptr(), pairs_lat=5, pairs_lon=6)
    assert sna._lib.sna_norm_rotate_forward(part, 1, sna.SNA_BFLOAT16, 2, 24, 0.5, 0, stream) == 0
    assert torch.equal(a, y)
    part.x, part.dy, part.dx = t(x), t(b), t(b)
    assert sna._lib.sna_norm_rotate_backward(part, 1, sna.SNA_BFLOAT16, 2, 24, 0.5, 0, None, 0, stream) == 0
    assert torch.equal(b, dx)


def test_gradient_against_differences():
    torch.manual_seed(3)
    q, k = (torch.randn(1, 2, 3, 4, 8, device="cuda") for _ in range(2))
    w = torch.randn(8, device="cuda")
    rotation = tables(3, 4, 2, 2)
    g = torch.randn(1, 2, 3, 4, 8, device="cuda")
    value = lambda q_, w_: (layer.qk_norm_rotate(q_, k, w_, None, rotation, rotation)[0].double() * g).sum()
    ends = [q.clone().requires_grad_(), w.clone().requires_grad_()]
    grads = torch.autograd.grad(value(*ends).float(), ends)
    step = 2.0 ** -7        # error of the central difference: step^2 / 6 of a third derivative, and 2^-24 of the values over 2 step
    for end, grad in zip((0, 1), grads):
        for index in [(0, 1, 2, 3, 5), (0, 0, 0, 0, 0), (0, 1, 1, 1, 7)]:
            at = index if end == 0 else index[-1:]
            shifted = []
            for sign in (1, -1):
                args = [q.clone(), w.clone()]
                args[end][at] += sign * step
                shifted.append(float(value(*args)))
            assert abs((shifted[0] - shifted[1]) / (2 * step) - float(grad[at])) < 5e-3


def test_without_weights_rotation_and_gradient():
    torch.manual_seed(0)
    q, k = heads(2, 3, 4, 5, 16, torch.float32).requires_grad_(), heads(2, 3, 4, 5, 16, torch.float32)
    out = layer.qk_norm_rotate(q, k)
    for x, y in zip((q, k), out):
        ref, size = definition(x.detach(), None, None, 1e-6, False)
        near(y.detach(), ref, size, 32, torch.float32, "out")
    assert torch.autograd.grad(out[0].sum(), q)[0].shape == q.shape      # (the other output takes no part)
    with torch.no_grad():
        assert not layer.qk_norm_rotate(q, k)[0].requires_grad


def test_rotated_scores_depend_on_the_difference_of_longitudes():
    torch.manual_seed(1)
    plan = sna.Plan(8, 24, 8, 24, 1, 1, 1.0, host_only=True)
    rotation, _ = layer.plan_rotations(plan, 32)
    x = torch.randn(2, 32, device="cuda")
    q, k = (v.expand(1, 1, 8, 24, 32) for v in x)
    q, k = layer.qk_norm_rotate(q, k, q_rotation=rotation, k_rotation=rotation)
    scores = torch.einsum("jc,lc->jl", q[0, 0, 3].double(), k[0, 0, 3].double())
    for shift in (1, 7, 23):
        rolled = scores.roll((shift, shift), (0, 1))
        assert float((rolled - scores).abs().max()) < 64 * 32 * U32      # 32 products of numbers below 6, tables rounded to 32 bits


def test_values_that_are_not_finite_stay_in_their_vector():
    torch.manual_seed(2)
    q = heads(1, 2, 3, 5, 24, torch.bfloat16)
    ref = layer.qk_norm_rotate(q, q, q_rotation=tables(3, 5, 5, 6), k_rotation=tables(3, 5, 5, 6))[0]
    q = q.clone()
    q[0, 1, 2, 3, 4], q[0, 0, 1, 1, 23] = math.nan, math.inf
    out = layer.qk_norm_rotate(q, q, q_rotation=tables(3, 5, 5, 6), k_rotation=tables(3, 5, 5, 6))[0]
    assert out[0, 1, 2, 3].isnan().all()
    others = torch.ones(1, 2, 3, 5, dtype=torch.bool, device="cuda")
    others[0, 1, 2, 3] = others[0, 0, 1, 1] = False
    assert torch.equal(out[others], ref[others])


def test_empty_tensors():
    q, k = torch.randn(0, 2, 3, 4, 8, device="cuda"), torch.randn(0, 1, 0, 4, 8, device="cuda")
    w = torch.ones(8, device="cuda", requires_grad=True)
    out = layer.qk_norm_rotate(q, k, w, w)
    assert out[0].shape == q.shape and out[1].shape == k.shape
    assert torch.equal(torch.autograd.grad(out[0].sum() + out[1].sum(), w)[0], torch.zeros(8, device="cuda"))


def test_another_stream_and_a_captured_graph():
    torch.manual_seed(4)
    q, k = heads(1, 2, 16, 33, 32, torch.bfloat16).requires_grad_(), heads(1, 2, 16, 33, 32, torch.bfloat16).requires_grad_()
    w = torch.rand(32, device="cuda").requires_grad_()
    rotation = tables(16, 33, 8, 8)

    def step():
        out = layer.qk_norm_rotate(q, k, w, w, rotation, rotation)
        # (a graph of the same leaves that lives on would make PyTorch's own accumulation of w's gradients wait for a stream outside the capture)
        return tuple(t.detach() for t in (*out, *torch.autograd.grad(out, (q, k, w), out)))

    ref = step()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        other = step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    with torch.no_grad():
        q.copy_(torch.randn_like(q))
    graph.replay()
    ref = step()
    assert all(torch.equal(a, b) for a, b in zip(ref, captured))


def test_refusals():
    q, k, w = heads(1, 2, 3, 4, 16, torch.float32), heads(1, 2, 3, 4, 16, torch.float32), torch.ones(16, device="cuda")
    rotation = tables(3, 4, 4, 4)
    call = layer.qk_norm_rotate
    for args, says in [((q[0], k), "B, H, nlat"), ((q.double(), k), "float32, bfloat16"), ((q, k.half()), "type of q"), ((q, k[..., :8]), "C = 16"),
                       ((q, k.cpu()), "CUDA tensor"), ((q.cpu(), k), "CUDA tensor"), ((q, k, w.half()), "q_weight"), ((q, k, None, w[:8]), "k_weight"),
                       ((q, k, None, None, tables(4, 4, 4, 4)), "table of latitudes"), ((q, k, None, None, tables(3, 5, 4, 4)), "table of longitudes"),
                       ((q, k, None, None, tables(3, 4, 5, 4)), "more pairs"), ((q, k, None, None, [t.double() for t in rotation]), "float32"),
                       ((q, torch.cat((k, k)),), "B = 1")]:
        with pytest.raises(ValueError, match=says):
            call(*args)
    with pytest.raises(sna.SnaError, match="multiple of 4"):
        call(q[..., :6], k[..., :6])
    with pytest.raises(sna.SnaError, match="eps"):
        call(q, k, eps=-1.0)
    with pytest.raises(ValueError, match="plain torch.Tensor"):
        call(q.as_subclass(type("Sub", (torch.Tensor,), {})), k)
    q.requires_grad_()
    out = call(q, k)[0]
    with pytest.raises(RuntimeError, match="differentiable once"):
        torch.autograd.grad(out.sum(), q, create_graph=True)


@pytest.mark.parametrize("saved", range(8), ids=["q", "k", "q_weight", "k_weight", "q_lat", "q_lon", "k_lat", "k_lon"])
@pytest.mark.parametrize("change, says", [(lambda t: t.cpu(), "CUDA tensor"), (lambda t: t.double(), "must be|type of"), (lambda t: t[:-1], "shape|must be"), (lambda t: t + 0, None)],
                         ids=["host", "double", "shape", "copy"])
def test_saved_tensors_that_hooks_return_are_checked(saved, change, says):
    torch.manual_seed(15)
    q, k = heads(2, 2, 3, 4, 16, torch.float32).requires_grad_(), heads(2, 1, 5, 6, 16, torch.float32).requires_grad_()
    w = [torch.randn(16, device="cuda").requires_grad_() for _ in range(2)]
    rotations = [tables(3, 4, 2, 3), tables(5, 6, 2, 3)]
    seen = []

    def unpack(t):
        seen.append(t)
        return change(t) if len(seen) == saved + 1 else t

    call = lambda: sum(o.square().sum() for o in layer.qk_norm_rotate(q, k, *w, *rotations))
    ref = torch.autograd.grad(call(), (q, k, *w))
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t):
        out = layer.qk_norm_rotate(q, k, *w, *rotations)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, unpack):
        out = layer.qk_norm_rotate(q, k, *w, *rotations)
    total = sum(o.square().sum() for o in out)
    if says:
        with pytest.raises(ValueError, match=says):
            torch.autograd.grad(total, (q, k, *w))
    else:
        assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(total, (q, k, *w)), ref))


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda d: str(d).split(".")[1])
@pytest.mark.parametrize("eps", [0.0, 1e-50])
@pytest.mark.parametrize("grid, C, interleaved", [((7, 13), 32, False), ((7, 13), 32, True), ((45, 90), 24, False), ((3, 5), 100, True), ((1, 1), 4, False), ((91, 180), 128, False)])
def test_gradients_without_eps(grid, C, interleaved, eps, dtype):
    """eps = 0, or below what 32 bits hold, on grids whose last block of points is not full."""
    torch.manual_seed(C)
    q, k = heads(2, 3, *grid, C, dtype).requires_grad_(), heads(2, 1, *grid, C, dtype).requires_grad_()
    weights = [torch.randn(C, device="cuda").requires_grad_() for _ in range(2)]
    pairs = (1, 1) if C == 100 else (C // 4, C // 4)        # (24 and 100 channels: pairs at a distance that is no multiple of a lane's, channels of no pair)
    rotation = tables(*grid, *pairs)
    out = layer.qk_norm_rotate(q, k, *weights, rotation, rotation, eps=eps, interleaved=interleaved)
    grads_out = [torch.randn(o.shape, device="cuda").to(dtype) for o in out]
    got = torch.autograd.grad(out, (q, k, *weights), grads_out)
    for i, (x, weight, g) in enumerate(zip((q, k), weights, grads_out)):
        ends = [x.detach().double().requires_grad_(), weight.detach().double().requires_grad_()]
        ref, size = definition(*ends, rotation, 0.0, interleaved)
        near(out[i].detach(), ref.detach(), size.detach(), C + 16, dtype, f"out {i}")
        ref_x, ref_w = torch.autograd.grad(ref, ends, g.double())
        xd = x.detach().double()
        r = 1 / xd.square().mean(-1, keepdim=True).sqrt()
        turned = definition_transposed_size(g.double(), rotation, interleaved)
        gw = turned * weight.detach().double().abs()
        near(got[i], ref_x, r * (gw + xd.abs() * r * (gw * xd.abs() * r).mean(-1, keepdim=True)), 3 * C + 32, dtype, f"dx {i}")
        near(got[2 + i], ref_w, (turned * xd.abs() * r).sum((0, 1, 2, 3)), C + 16 + x.numel() // C, torch.float32, f"dw {i}")


@pytest.mark.parametrize("C, pairs, interleaved", [(32, (8, 8), False), (64, (16, 16), True), (24, (5, 6), False)], ids=["by shuffle", "within a lane", "by shared memory"])
def test_results_in_place_of_inputs_for_all_pairs(C, pairs, interleaved):
    torch.manual_seed(12)
    x, w, g = heads(3, 5, 7, 9, C, torch.float16), torch.randn(C, device="cuda"), heads(3, 5, 7, 9, C, torch.float16)
    rotation = tables(7, 9, *pairs)
    xr, wr = x.clone().requires_grad_(), w.clone().requires_grad_()
    y = layer.qk_norm_rotate(xr, xr.detach(), wr, w, rotation, rotation, interleaved=interleaved)[0]
    dx, dw = torch.autograd.grad(y, (xr, wr), g)
    t = lambda a: sna.SnaTensor(a.data_ptr(), a.stride(0), a.stride(1), a.stride(2), a.stride(3))
    stream = torch.cuda.current_stream().cuda_stream
    a, b, dw2 = x.clone(), g.clone(), torch.empty_like(w)
    part = sna.SnaRotate(nlat=7, nlon=9, H=5, x=t(a), y=t(a), weight=w.data_ptr(), lat_table=rotation[0].data_ptr(), lon_table=rotation[1].data_ptr(), pairs_lat=pairs[0], pairs_lon=pairs[1])
    assert sna._lib.sna_norm_rotate_forward(part, 1, sna.SNA_FLOAT16, 3, C, 1e-6, interleaved, stream) == 0
    assert torch.equal(a, y)
    part.x, part.dy, part.dx, part.dweight = t(x), t(b), t(b), dw2.data_ptr()
    need = sna._lib.sna_norm_rotate_workspace_bytes(C)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    assert sna._lib.sna_norm_rotate_backward(part, 1, sna.SNA_FLOAT16, 3, C, 1e-6, interleaved, ws.data_ptr(), need, stream) == 0
    assert torch.equal(b, dx) and torch.equal(dw2, dw)
