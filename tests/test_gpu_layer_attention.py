"""16-bit attention with weights per point against its definition in 64 bits: types, head widths, shared heads, strides, points left out, rows
without points, few queries, splits over keys, gradients."""
import math

import pytest
import torch

from paper_2505_11157_b200 import layer, sna

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16]
U32 = 2.0 ** -24


def heads(B, H, grid, C, dtype, order="plain", scale=1.0):
    nlat, nlon = grid
    r = lambda *shape: (scale * torch.randn(*shape, device="cuda")).to(dtype)
    if order == "plain":
        return r(B, H, nlat, nlon, C)
    if order == "points first":
        return r(B, nlat, nlon, H, C).permute(0, 3, 1, 2, 4)
    if order == "packed":
        return r(B, nlat, nlon, 3, H, C)[:, :, :, 1].permute(0, 3, 1, 2, 4)
    if order == "shared":
        return r(B, 1, nlat, nlon, C).expand(B, H, nlat, nlon, C)
    if order == "rows apart":               # rings with a gap between them: not in one line
        return r(B, H, nlat, nlon + 3, C)[:, :, :, :nlon]
    if order == "odd":
        return r(B, H, nlat, nlon, C + 4)[..., 4:]
    raise AssertionError(order)


def reference(q, k, v, weights, scale, dout):
    """Values and gradients in 64 bits, and how far off the operator may be (see each bound)."""
    dtype = q.dtype
    u = torch.finfo(dtype).eps / 2
    half = dtype == torch.float16
    B, Hq = q.shape[:2]
    Hk, C = k.shape[1], k.shape[-1]
    flat = lambda x: x.detach().double().reshape(B, Hk, -1, C)      # (of queries: the heads of a group, one below the other)
    Q, Y, K, V = flat(q), flat(dout), flat(k), flat(v)
    Nk = K.shape[2]
    w = torch.zeros(B, 1, 1, Nk, dtype=torch.float64, device="cuda") if weights is None else weights.double().reshape(-1, 1, 1, Nk).expand(B, 1, 1, Nk)
    out_of = w <= -1e30
    K, V = torch.where(out_of.transpose(2, 3), 0.0, K), torch.where(out_of.transpose(2, 3), 0.0, V)
    w = torch.where(out_of, -math.inf, w)
    s = Q @ K.transpose(2, 3) * scale + w
    top = s.amax(-1, keepdim=True) if Nk else torch.full((*s.shape[:3], 1), -math.inf, dtype=torch.float64, device="cuda")
    e = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(-1, keepdim=True)
    p = e / torch.where(total == 0, 1.0, total)
    lse = (top + total.log()).squeeze(-1)
    out = p @ V
    t = Y @ V.transpose(2, 3)
    D = (Y * out).sum(-1, keepdim=True)
    ds = p * (t - D)
    grads = [scale * ds @ K, scale * ds.transpose(2, 3) @ Q, p.transpose(2, 3) @ Y]
    # relative error of a probability: that of its score (C products and sums in 32 bits, the weight, the scale to base 2), once for itself, the
    # row's maximum and the sum; exp2 in hardware adds 2^-22
    finite = lambda x: torch.where(x == -math.inf, 0.0, x).abs().max().item() if x.numel() else 0.0
    size = (abs(scale) * (Q.abs() @ K.abs().transpose(2, 3)).max().item() if Nk and Q.shape[2] else 0.0) + finite(w)
    dp = 3 * ((C + 8) * 2 * U32 * size + 2.0 ** -22)
    many = 2 * U32 * max(Nk, Q.shape[2])          # sums of products in 32 bits (the tensor cores may truncate)
    # float16 operands, held times 2^14, end at 2^-24 in steps; exp2 in hardware gives zero below 2^-126, which is all that bounds a bfloat16 operand
    least = 2.0 ** -38 if half else 2.0 ** -126
    tol_out = (p @ V.abs()) * (u + 2 * dp + many) + least * V.abs().sum(2, keepdim=True) + u * (1 + u) * out.abs()
    dD = (Y.abs() * (u * out.abs() + tol_out)).sum(-1, keepdim=True) + C * 2 * U32 * (Y.abs() * out.abs()).sum(-1, keepdim=True)
    dt = C * 2 * U32 * (Y.abs() @ V.abs().transpose(2, 3))
    bound = 2 * Y.norm(dim=-1).amax().item() * V.norm(dim=-1).amax().item() if Nk and Q.shape[2] else 0.0
    tol_ds = p * ((t - D).abs() * (u + 2 * dp + many) + dD + dt) + 2 * least * bound
    tols = [abs(scale) * tol_ds @ K.abs() + u * (1 + u) * grads[0].abs(), abs(scale) * tol_ds.transpose(2, 3) @ Q.abs() + u * (1 + u) * grads[1].abs(),
            p.transpose(2, 3) @ Y.abs() * (u + 2 * dp + many) + least * Y.abs().sum(2, keepdim=True) + u * (1 + u) * grads[2].abs()]
    values = [out.reshape(q.shape), grads[0].reshape(q.shape), grads[1].reshape(k.shape), grads[2].reshape(k.shape)]
    tols = [x.reshape(y.shape) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps for x, y in zip([tol_out, *tols], values)]
    return values, tols, lse.reshape(q.shape[:4]), dp + many


def close(got, ref, tol, what):
    off = (got.double() - ref).abs()
    assert got.shape == ref.shape and bool((off <= tol).all()), (what, float((off / tol).max()))


def check(q, k, v, weights=None, scale=None, dout_order="plain"):
    q, k, v = (x.detach().requires_grad_() for x in (q, k, v))
    out, lse = layer.weighted_attention(q, k, v, weights, scale, return_lse=True)
    dout = heads(*q.shape[:2], q.shape[2:4], q.shape[4], q.dtype, dout_order)
    grads = torch.autograd.grad(out, (q, k, v), dout, retain_graph=True)
    again = torch.autograd.grad(out, (q, k, v), dout)
    values, tols, lse_ref, d_lse = reference(q, k, v, weights, q.shape[-1] ** -0.5 if scale is None else scale, dout)
    for name, got, ref, tol in zip(("out", "dq", "dk", "dv"), (out.detach(), *grads), values, tols):
        assert got.dtype == q.dtype
        close(got, ref, tol, name)
    empty = lse_ref == -math.inf
    assert torch.equal(lse == -math.inf, empty)
    close(torch.where(empty, 0.0, lse), torch.where(empty, 0.0, lse_ref), d_lse + 4 * U32 * lse_ref.abs().masked_fill(empty, 0.0), "lse")
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
    with torch.no_grad():
        assert torch.equal(layer.weighted_attention(q, k, v, weights, scale), out)
    return out, lse, grads


CASES = [
    # B, Hq, Hk, q grid, k grid, C, order
    (1, 1, 1, (1, 1), (1, 1), 8, "plain"),
    (2, 2, 2, (5, 9), (5, 9), 32, "plain"),
    (2, 4, 2, (7, 13), (14, 26), 64, "points first"),
    (3, 6, 2, (3, 67), (9, 15), 24, "packed"),
    (1, 5, 1, (33, 17), (2, 301), 128, "plain"),
    (2, 8, 2, (1, 1), (31, 67), 64, "plain"),
    (1, 3, 3, (1, 16), (1, 63), 40, "rows apart"),
    (1, 4, 4, (1, 17), (1, 65), 80, "odd"),
    (2, 2, 1, (16, 8), (8, 8), 96, "rows apart"),
    (1, 2, 2, (16, 33), (33, 16), 16, "shared"),
    (1, 8, 1, (1, 2), (90, 181), 32, "points first"),
    (1, 1, 1, (128, 1), (1, 128), 128, "plain"),
    (1, 2, 2, (45, 90), (45, 90), 64, "plain"),
    (2, 4, 1, (20, 41), (23, 45), 128, "packed"),
]


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda d: str(d).split(".")[1])
@pytest.mark.parametrize("weights", ["none", "shared", "per field"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_values_and_gradients(case, weights, dtype):
    B, Hq, Hk, q_grid, k_grid, C, order = case
    torch.manual_seed(C + B)
    q, k, v = heads(B, Hq, q_grid, C, dtype, order), heads(B, Hk, k_grid, C, dtype, order), heads(B, Hk, k_grid, C, dtype, order)
    points = k_grid[0] * k_grid[1]
    w = None if weights == "none" else torch.randn(points if weights == "shared" else (B, points), device="cuda")
    check(q, k, v, w, dout_order="points first" if order == "plain" else "plain")


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda d: str(d).split(".")[1])
@pytest.mark.parametrize("Nq, C", [(1, 32), (3, 128), (150, 64), (150, 128), (300, 32)])
@pytest.mark.parametrize("low", [-math.inf, torch.finfo(torch.float32).min, float(torch.finfo(torch.bfloat16).min), -1e30])
def test_points_left_out_may_hold_anything(dtype, Nq, C, low):
    torch.manual_seed(Nq)
    B, Hq, Hk, grid = 4, 4, 2, (7, 93)
    q, k, v = heads(B, Hq, (1, Nq), C, dtype), heads(B, Hk, grid, C, dtype), heads(B, Hk, grid, C, dtype)
    w = torch.randn(B, 7 * 93, device="cuda")
    gone = torch.rand(B, 7 * 93, device="cuda") < 0.3
    gone[1] = True                          # a field without any point
    gone[2, :200] = True                    # whole blocks at the start and the end
    gone[2, -200:] = True
    gone[3] = True
    gone[3, 333] = False                    # a single point
    w[gone] = low
    clean = check(q, k, v, w)
    assert not clean[0][1].any() and bool((clean[1][1] == -math.inf).all()) and not any(bool(g[1].any()) for g in clean[2])
    for value in (math.nan, math.inf):
        k2, v2 = (x.clone() for x in (k, v))
        for x in (k2, v2):
            x.masked_fill_(gone.reshape(B, 1, 7, 93, 1), value)
        torch.manual_seed(Nq + 1)
        ref = run(q, k, v, w)
        torch.manual_seed(Nq + 1)
        got = run(q, k2, v2, w)
        assert all(torch.equal(a, b) for a, b in zip(ref, got))


def run(q, k, v, w=None):
    ends = [x.detach().requires_grad_() for x in (q, k, v)]
    out = layer.weighted_attention(*ends, w)
    return (out.detach(), *torch.autograd.grad(out, ends, torch.randn(q.shape, device="cuda").to(q.dtype)))


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda d: str(d).split(".")[1])
@pytest.mark.parametrize("C", [32, 64, 128])
def test_peaked_flat_and_small_data(dtype, C):
    torch.manual_seed(C)
    grid = (20, 41)
    q, k, v = (heads(1, 2, grid, C, dtype) for _ in range(3))
    check(q, k, v, scale=4.0)                                   # almost one point per row
    check(q, k, v, scale=0.0)                                   # all points alike
    check(q, k, v, scale=-0.3)
    check(q, k, v, torch.linspace(0, 90, 820, device="cuda"))   # later blocks outweigh earlier ones by far
    check(q, k, v, torch.linspace(90, 0, 820, device="cuda"))
    small = 2.0 ** -10
    check(q, k, v * small)
    check(q, k * small, v)


def test_float16_gradients_of_small_size_keep_their_digits():
    """dout of 2^-13 over thousands of points: ds is far below the smallest float16 number but for the scale it is held times."""
    torch.manual_seed(5)
    q, k, v = (heads(1, 1, (50, 100), 32, torch.float16) for _ in range(3))
    ends = [x.detach().requires_grad_() for x in (q, k, v)]
    out = layer.weighted_attention(*ends)
    dout = (torch.randn(out.shape, device="cuda") * 2.0 ** -3).half()
    ref = torch.autograd.grad(out, ends, dout, retain_graph=True)
    got = torch.autograd.grad(out, ends, dout * 2.0 ** -8)
    for a, b in zip(ref, got):
        # (the results themselves are rounded to float16's smallest steps, half of 2^-24)
        assert bool(((a.double() * 2.0 ** -8 - b.double()).abs() <= 2.0 ** -10 * b.double().abs() + 2.0 ** -24).all())


def test_values_that_are_not_finite_reach_their_rows():
    torch.manual_seed(6)
    for Nq in (3, 200):
        q, k, v = (heads(1, 2, (1, n), 64, torch.bfloat16) for n in (Nq, 300, 300))
        ref = run(q, k, v)[0]
        q[0, 1, 0, 2, 5] = math.nan
        torch.manual_seed(1)
        out = run(q, k, v)[0]
        assert out[0, 1, 0, 2].isnan().all() and torch.equal(out[0, 0], ref[0, 0]) and not out[0, 1, 0, :2].isnan().any()
        v[0, 0, 0, 7, 3] = math.nan
        out = run(q, k, v)[0]
        assert out[0, 0, 0, :, 3].isnan().all() and torch.equal(out[0, 0, 0, :, 4:], ref[0, 0, 0, :, 4:])


def test_gradient_against_differences():
    torch.manual_seed(7)
    q, k, v = (heads(1, 2, (3, 5), 16, torch.float16) for _ in range(3))
    w = torch.randn(15, device="cuda")
    g = torch.randn(q.shape, device="cuda").half()
    value = lambda *x: float((layer.weighted_attention(*x, w).double() * g.double()).sum())
    ends = [x.clone().requires_grad_() for x in (q, k, v)]
    grads = torch.autograd.grad(layer.weighted_attention(*ends, w), ends, g)
    step = 2.0 ** -4        # exact in float16; rounding of 480 outputs (2^-12 each, in a random order) over 2 step, and step^2 / 6 of a third derivative
    for i in range(3):
        for index in [(0, 0, 1, 2, 3), (0, 1, 2, 4, 15)]:
            sides = []
            for sign in (1, -1):
                x = [q.clone(), k.clone(), v.clone()]
                x[i][index] += sign * step
                sides.append((value(*x), float(x[i][index])))
            assert abs((sides[0][0] - sides[1][0]) / (sides[0][1] - sides[1][1]) - float(grads[i][index])) < 0.08


def test_global_attention_of_a_plan_agrees_with_the_fp32_operator():
    torch.manual_seed(8)
    plan = sna.Plan(16, 32, 8, 16, 0, 0, global_attention=True)
    q, k, v = heads(2, 2, (8, 16), 32, torch.bfloat16), heads(2, 2, (16, 32), 32, torch.bfloat16), heads(2, 2, (16, 32), 32, torch.bfloat16)
    ref = plan.forward(*(x.float() for x in (q, k, v)))
    out = layer.weighted_attention(q, k, v, layer.log_quadrature_weights(plan))
    values, tols, _, _ = reference(q, k, v, layer.log_quadrature_weights(plan), 32 ** -0.5, torch.zeros_like(q))
    close(out, ref.double(), tols[0] + 1e-5 * float(ref.abs().max()), "out")


def test_empty_sizes():
    for q_shape, k_shape in [((0, 2, 3, 4, 16), (0, 1, 5, 6, 16)), ((2, 2, 0, 4, 16), (2, 1, 5, 6, 16)), ((2, 2, 3, 4, 16), (2, 1, 5, 0, 16)), ((2, 0, 3, 4, 16), (2, 0, 5, 6, 16))]:
        q = torch.randn(q_shape, device="cuda").bfloat16().requires_grad_()
        k, v = (torch.randn(k_shape, device="cuda").bfloat16().requires_grad_() for _ in range(2))
        out, lse = layer.weighted_attention(q, k, v, return_lse=True)
        assert out.shape == q.shape and not out.any() and bool((lse == -math.inf).all())
        assert not any(bool(g.any()) for g in torch.autograd.grad(out.sum(), (q, k, v)))


def test_rows_behind_a_result_stay_as_they_were():
    """Through the C ABI: outputs that are slices of larger tensors."""
    torch.manual_seed(9)
    B, H, N, C = 2, 3, 100, 40
    q, k, v, y = (heads(B, H, (1, N), C, torch.bfloat16) for _ in range(4))
    big = [torch.full((B, H + 1, 1, N + 5, C + 8), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(4)]
    part = [x[:, :H, :, :N, :C] for x in big]
    describe = lambda t: sna.SnaTensor(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2), t.stride(3))
    lse = torch.empty(B, H, N, device="cuda")
    a = sna.SnaAttention(B=B, Hq=H, Hk=H, C=C, nlat_q=1, nlon_q=N, nlat_k=1, nlon_k=N, q=describe(q), k=describe(k), v=describe(v), out=describe(part[0]), lse=lse.data_ptr(), scale=0.2)
    need = sna._lib.sna_attention_forward_workspace_bytes(a, 1)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    assert sna._lib.sna_attention_forward(a, 1, ws.data_ptr(), need, stream) == 0
    a.dout, a.dq, a.dk, a.dv = describe(y), *(describe(t) for t in part[1:])
    need = sna._lib.sna_attention_backward_workspace_bytes(a, 1)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    assert sna._lib.sna_attention_backward(a, 1, ws.data_ptr(), need, stream) == 0
    values, tols, _, _ = reference(q, k, v, None, 0.2, y)
    for x, inside, ref, tol in zip(big, part, values, tols):
        close(inside, ref, tol, "slice")
        inside.fill_(7.0)
        assert bool((x == 7.0).all())


@pytest.mark.parametrize("Nq", [4, 300])
def test_another_stream_and_a_captured_graph(Nq):
    torch.manual_seed(10)
    q, k, v = (heads(2, 2, (1, n), 64, torch.float16).requires_grad_() for n in (Nq, 700, 700))
    w = torch.randn(700, device="cuda")
    g = torch.randn(q.shape, device="cuda").half()

    def step():
        out = layer.weighted_attention(q, k, v, w)
        return tuple(t.detach() for t in (out, *torch.autograd.grad(out, (q, k, v), g)))

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
        for x in (q, k, v):
            x.copy_(torch.randn_like(x))
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(step(), captured))


def test_refusals():
    q, k, v = (heads(2, 4, (3, 4), 16, torch.bfloat16) for _ in range(3))
    w = torch.zeros(12, device="cuda")
    call = layer.weighted_attention
    for args, says in [((q[0], k, v), "B, H, nlat"), ((q.float(), k, v), "bfloat16 or float16"), ((q, k.half(), v), "type of q"), ((q, k, v[:, :2]), "v has shape"),
                       ((q, k[..., :8], v[..., :8]), "C = 16"), ((q, k[:, :3], v[:, :3]), "multiple of k's"), ((q, k.cpu(), v), "CUDA tensor"), ((q.cpu(), k, v), "CUDA tensor"),
                       ((q, k[:1], v[:1]), "B = 2"), ((q, k, v, w[:11]), "log_weights"), ((q, k, v, w.half()), "float32"), ((q, k, v, w.cpu()), "CUDA tensor"),
                       ((q, k, v, w.expand(3, 12)), "log_weights"), ((q, k, v, w.clone().requires_grad_()), "no gradient")]:
        with pytest.raises(ValueError, match=says):
            call(*args)
    with pytest.raises(sna.SnaError, match="multiple of 8"):
        call(*(x[..., :12] for x in (q, k, v)))
    with pytest.raises(sna.SnaError, match="scale"):
        call(q, k, v, scale=math.inf)
    with pytest.raises(ValueError, match="plain torch.Tensor"):
        call(q.as_subclass(type("Sub", (torch.Tensor,), {})), k, v)
    q.requires_grad_()
    out = call(q, k, v)
    with pytest.raises(RuntimeError, match="differentiable once"):
        torch.autograd.grad(out.sum(), q, create_graph=True)


def test_no_kernel_gave_up_on_a_wait():
    """Last in this file: every bounded wait of the calls above came to its end."""
    sna.sna_layer_check()


def test_a_wait_that_runs_out_is_reported_once():
    sna.sna_layer_check()
    sna.sna_debug_exercise_layer_wait()
    with pytest.raises(sna.SnaError, match="gave up on a bounded wait"):
        sna.sna_layer_check()
    sna.sna_layer_check()
    after = run(*(heads(1, 1, (1, 200), 32, torch.bfloat16) for _ in range(3)))
    assert all(bool(torch.isfinite(t).all()) for t in after)


@pytest.mark.parametrize("saved", range(7), ids=["q", "k", "v", "log_weights", "out", "lse", "rest"])
@pytest.mark.parametrize("change, says", [(lambda t: t.cpu(), "CUDA tensor"), (lambda t: t.double(), "must be|type of q"), (lambda t: t[..., :-1], "shape|must be|C ="),
                                          (lambda t: t + 0, None), (lambda t: t.transpose(0, 1).contiguous().transpose(0, 1) if t.dim() == 5 else t, None)],
                         ids=["host", "double", "shape", "copy", "strides"])
def test_saved_tensors_that_hooks_return_are_checked(saved, change, says):
    torch.manual_seed(12)
    q, k, v = (heads(2, 2, (1, n), 32, torch.bfloat16).requires_grad_() for n in (20, 70, 70))
    w = torch.randn(2, 70, device="cuda")
    g = torch.randn(q.shape, device="cuda").bfloat16()
    seen = []

    def unpack(t):
        seen.append(t)
        return change(t) if len(seen) == saved + 1 else t

    ref = torch.autograd.grad(layer.weighted_attention(q, k, v, w), (q, k, v), g)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, unpack):
        out = layer.weighted_attention(q, k, v, w)
    if says:
        with pytest.raises(ValueError, match=says):
            torch.autograd.grad(out, (q, k, v), g)
    else:
        assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out, (q, k, v), g), ref))
    assert len(seen) == 7


def test_inputs_changed_before_the_backward_pass_and_single_gradients():
    torch.manual_seed(13)
    q, k, v = (heads(1, 2, (1, 90), 32, torch.float16) for _ in range(3))
    ends = [x.clone().requires_grad_() for x in (q, k, v)]
    g = torch.randn(q.shape, device="cuda").half()
    ref = torch.autograd.grad(layer.weighted_attention(*ends), ends, g)
    for i in range(3):
        ends = [x.clone().requires_grad_(j == i) for j, x in enumerate((q, k, v))]
        assert torch.equal(torch.autograd.grad(layer.weighted_attention(*ends), ends[i], g)[0], ref[i])
    ends = [x.clone().requires_grad_() for x in (q, k, v)]
    w = torch.zeros(90, device="cuda")
    out = layer.weighted_attention(*ends, w)
    w += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


def test_threads_and_streams_at_once():
    import threading
    torch.manual_seed(14)
    inputs = [[heads(1, 4, (1, n), 64, torch.bfloat16) for _ in range(3)] for n in (200, 700, 90, 8)]
    refs = []
    for x in inputs:
        torch.manual_seed(1)
        refs.append(run(*x))
    torch.cuda.synchronize()
    results = [None] * len(inputs)

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            gens = [t.detach().requires_grad_() for t in inputs[i]]
            for _ in range(20):
                out = layer.weighted_attention(*gens)
                results[i] = (out.detach(), *torch.autograd.grad(out, gens, torch.ones_like(out)))
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(inputs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for x, got, ref in zip(inputs, results, refs):
        assert torch.equal(got[0], ref[0])
        gens = [t.detach().requires_grad_() for t in x]
        out = layer.weighted_attention(*gens)
        assert all(torch.equal(a, b) for a, b in zip(got[1:], torch.autograd.grad(out, gens, torch.ones_like(out))))


def test_saved_weights_that_hooks_return_with_other_strides():
    # (every layout below lies within memory of as many values as are read from it)
    torch.manual_seed(16)
    q, k, v = (heads(2, 2, (1, n), 32, torch.bfloat16).requires_grad_() for n in (20, 70, 70))
    w = torch.randn(2, 70, device="cuda")
    g = torch.randn(q.shape, device="cuda").bfloat16()
    ref = torch.autograd.grad(layer.weighted_attention(q, k, v, w), (q, k, v), g)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t.t().contiguous().t() if t.shape == w.shape else t):
        out = layer.weighted_attention(q, k, v, w)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out, (q, k, v), g), ref))


@pytest.mark.parametrize("n", [8, 200])
@pytest.mark.parametrize("weighted", [False, True])
def test_a_row_of_nan_says_so_in_its_lse(n, weighted):
    torch.manual_seed(17)
    q, k, v = heads(1, 1, (1, n), 32, torch.bfloat16), heads(1, 1, (1, 200), 32, torch.bfloat16), heads(1, 1, (1, 200), 32, torch.bfloat16)
    q[0, 0, 0, 3, 5] = math.nan
    w = torch.randn(200, device="cuda") if weighted else None
    out, lse = layer.weighted_attention(q, k, v, w, return_lse=True)
    nan = torch.arange(n, device="cuda") == 3
    assert torch.equal(lse[0, 0, 0].isnan(), nan) and torch.equal(out[0, 0, 0].isnan().all(-1), nan) and torch.equal(out[0, 0, 0].isnan().any(-1), nan)


@pytest.mark.parametrize("axes", [(2, 3), (3,), (0, 2, 3), (1,)])
def test_gradients_of_means(axes):
    torch.manual_seed(18)
    ends = [heads(2, 2, (3, n), 32, torch.bfloat16).requires_grad_() for n in (30, 40, 40)]
    out = layer.weighted_attention(*ends)
    g = torch.randn(out.mean(axes, keepdim=True).shape, device="cuda").bfloat16()
    for got, ref in zip(torch.autograd.grad(out, ends, g.expand_as(out), retain_graph=True), torch.autograd.grad(out, ends, g.expand_as(out).contiguous())):
        assert torch.equal(got, ref)


def test_a_pending_negation_is_refused_and_that_of_a_gradient_taken():
    torch.manual_seed(19)
    q, k, v = (heads(1, 1, (1, 100), 32, torch.float16).requires_grad_() for _ in range(3))
    g = torch.randn(q.shape, device="cuda").half()
    pending = torch._neg_view(g)
    assert pending.is_neg()
    for args in ((pending, k, v), (q, pending, v), (q, k, pending)):
        with pytest.raises(ValueError, match="pending negation"):
            layer.weighted_attention(*args)
    with pytest.raises(ValueError, match="pending negation"):
        layer.qk_norm_rotate(q, pending)
    with pytest.raises(ValueError, match="pending negation"):
        layer.residual_dropout(pending, layer.dropout_state("cuda"), 0.5)
    w = torch.ones(32, device="cuda")
    state = layer.dropout_state("cuda")
    for f in (lambda: layer.weighted_attention(q, k, v), lambda: layer.qk_norm_rotate(q, k, w)[0], lambda: layer.residual_dropout(q, state, 0.5)):
        assert torch.equal(torch.autograd.grad(f(), q, pending)[0], torch.autograd.grad(f(), q, -g)[0])


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda d: str(d).split(".")[1])
@pytest.mark.parametrize("shape", [(3, 8, 2, 5500, 1030, 40), (2, 16, 2, 2100, 2049, 64), (12, 8, 4, 2000, 700, 128), (1, 16, 1, 135, 62200, 24), (20, 10, 2, 10600, 64, 8)],
                         ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("order", ["plain", "packed"])
@pytest.mark.parametrize("shared", [False, True], ids=["per field", "shared"])
def test_many_points_left_out(shape, dtype, order, shared):
    # the points that take part are brought together where a sixteenth of a field's or more is left out, if there is work enough (2^27 pairs of a row and a point):
    # fields on either side of that, without any points, with one, some or all of them
    B, Hq, Hk, Nq, Nk, C = shape
    torch.manual_seed(Nk)
    q, k, v = heads(B, Hq, (1, Nq), C, dtype, order), heads(B, Hk, (1, Nk), C, dtype, order), heads(B, Hk, (1, Nk), C, dtype, order)
    w = torch.randn(1 if shared else B, Nk, device="cuda")
    left = [Nk // 2, 0, Nk - Nk // 16 + 1, 1, Nk, min(Nk, 128), min(Nk, 129), 64, 1 + Nk // 3, Nk - Nk // 16]
    for case in range(0, len(left), 1 if shared else B):
        out_of = torch.ones(w.shape, dtype=torch.bool, device="cuda")
        for b in range(w.shape[0]):
            out_of[b, torch.randperm(Nk, device="cuda")[:left[(case + b) % len(left)]]] = False
        gone = out_of.expand(B, Nk)[:, None, None, :, None]
        kk, vv = k.masked_fill(gone, math.nan), v.masked_fill(gone, math.inf)
        out, lse, (dq, dk, dv) = check(q, kk, vv, w.masked_fill(out_of, -math.inf))
        assert not bool(dk.masked_select(gone).any()) and not bool(dv.masked_select(gone).any())
        none = out_of.all(1).expand(B)
        assert not bool(out[none].any()) and not bool(dq[none].any())


def test_rows_of_a_selection_in_a_captured_graph():
    # the same graph with other masks: nothing of the selection is decided on the host
    torch.manual_seed(21)
    B, H, N, C = 2, 4, 4200, 32
    ends = [heads(B, H, (1, N), C, torch.bfloat16).requires_grad_() for _ in range(3)]
    g = heads(B, H, (1, N), C, torch.bfloat16)
    w = torch.zeros(B, N, device="cuda")
    step = lambda: (lambda out: (out.detach(), *torch.autograd.grad(out, ends, g)))(layer.weighted_attention(*ends, w))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for share in (0.0, 0.5, 0.03, 1.0, 0.9):
        w.copy_(torch.randn(B, N, device="cuda").masked_fill(torch.rand(B, N, device="cuda") < share, -math.inf))
        graph.replay()
        got = [t.clone() for t in captured]
        assert all(torch.equal(a, b) for a, b in zip(got, step()))


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda d: str(d).split(".")[1])
@pytest.mark.parametrize("shape", [(2, 4, 2, 800, 1203, 8), (1, 2, 2, 900, 1100, 16), (1, 1, 1, 33, 9800, 32), (2, 2, 1, 300, 406, 64), (1, 2, 2, 260, 1000, 128), (1, 3, 3, 10, 40, 40)],
                         ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("weighted", [False, True])
def test_gradients_of_narrow_heads_and_small_problems_round_once(shape, weighted, dtype):
    # p and ds in two 16-bit parts: their second rounding is off by u^2 of the term (as is the product of the first's remainder and that), so that dv is off by half a
    # step of the result and what 32-bit sums and exponentials lose
    B, Hq, Hk, Nq, Nk, C = shape
    torch.manual_seed(Nk)
    q, k, v = heads(B, Hq, (1, Nq), C, dtype), heads(B, Hk, (1, Nk), C, dtype), heads(B, Hk, (1, Nk), C, dtype)
    w = torch.randn(Nk, device="cuda") if weighted else None
    check(q, k, v, w)
    dout = heads(B, Hq, (1, Nq), C, dtype)
    ends = [x.detach().requires_grad_() for x in (q, k, v)]
    dv = torch.autograd.grad(layer.weighted_attention(*ends, w), ends[2], dout)[0]
    values, _, _, d_lse = reference(q, k, v, w, C ** -0.5, dout)
    u = torch.finfo(dtype).eps / 2
    flat = lambda x: x.double().reshape(B, Hk, -1, C)
    s = flat(q) @ flat(k).transpose(2, 3) * C ** -0.5 + (0 if w is None else w.double())
    terms = (torch.softmax(s, -1).transpose(2, 3) @ flat(dout).abs()).reshape(dv.shape)
    least = 2.0 ** -38 if dtype == torch.float16 else 2.0 ** -126
    tol = terms * (2 * u * u + 2 * d_lse) + least * flat(dout).abs().sum(2, keepdim=True).reshape(B, Hk, 1, 1, C) + u * (1 + u) * values[3].abs()
    close(dv, values[3], tol, "dv")


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda d: str(d).split(".")[1])
@pytest.mark.parametrize("shape", [(1, 1, 1, 33, 9800, 32), (2, 4, 1, 17, 20011, 64), (1, 2, 2, 20011, 65, 40), (1, 4, 1, 9001, 130, 128), (2, 3, 3, 129, 5000, 96), (1, 16, 8, 9800, 64, 8)],
                         ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("share", [0.0, 0.5])
def test_long_and_narrow_problems(shape, share, dtype):
    # one side's tiles are cut into pieces, over whole ranges of points left out too
    B, Hq, Hk, Nq, Nk, C = shape
    torch.manual_seed(Nk)
    q, k, v = heads(B, Hq, (1, Nq), C, dtype), heads(B, Hk, (1, Nk), C, dtype), heads(B, Hk, (1, Nk), C, dtype)
    w = torch.randn(B, Nk, device="cuda").masked_fill(torch.rand(B, Nk, device="cuda") < share, -math.inf)
    w[0, Nk // 8: Nk // 8 + int(share * Nk)] = -math.inf
    check(q, k, v, w)


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda d: str(d).split(".")[1])
@pytest.mark.parametrize("weighted", [False, True])
def test_no_query_heads(weighted, dtype):
    q = torch.randn(2, 0, 3, 100, 32, device="cuda").to(dtype).requires_grad_()
    k, v = (torch.randn(2, 2, 20, 30, 32, device="cuda").to(dtype).requires_grad_() for _ in range(2))
    out = layer.weighted_attention(q, k, v, torch.randn(600, device="cuda") if weighted else None)
    assert out.shape == q.shape
    spoil = torch.full((2, 2, 20, 30, 32), math.nan, device="cuda", dtype=dtype)        # (what the next results' memory may hold)
    del spoil
    assert not any(bool(g.any()) for g in torch.autograd.grad(out.sum(), (q, k, v)))
