"""The layer's operators together, as the module runs them: against the same composition in 64 bits, in training, captured, under checkpointing."""
import copy
import math

import pytest
import torch

from paper_2505_11157_b200 import layer, sna
from paper_2505_11157_b200.module import SphericalNeighborhoodAttention

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def exact_convolutions():
    before = torch.backends.cudnn.allow_tf32, torch.backends.cuda.matmul.allow_tf32
    torch.backends.cudnn.allow_tf32 = torch.backends.cuda.matmul.allow_tf32 = False
    yield
    torch.backends.cudnn.allow_tf32, torch.backends.cuda.matmul.allow_tf32 = before


def rotate(x, rotation):
    lat, lon = (t.double() for t in rotation)
    angles = torch.cat((lat[:, None].expand(-1, lon.shape[0], -1, 2), lon[None].expand(lat.shape[0], -1, -1, 2)), 2)
    pairs = angles.shape[2]
    a, b, cos, sin = x[..., :pairs], x[..., pairs:2 * pairs], angles[..., 0], angles[..., 1]
    return torch.cat((a * cos - b * sin, a * sin + b * cos, x[..., 2 * pairs:]), -1)


def plain(m, x_q, x_kv, residual=None):
    """The module in 64 bits: every point attends to every point with its quadrature weight."""
    P = {name: p.double() for name, p in m.named_parameters()}
    heads = lambda x, w, b: torch.nn.functional.conv2d(x, w, b).unflatten(1, (m.heads, m.head_dim)).permute(0, 1, 3, 4, 2)
    q, k, v = heads(x_q, P["wq"], P["bq"]), heads(x_kv, P["wk"], P["bk"]), heads(x_kv, P["wv"], P["bv"])
    rotations = layer.plan_rotations(m.plan, m.head_dim) if m.rotary else (None, None)
    if m.qk_norm or m.rotary:
        new = []
        for x, name, rotation in ((q, "q_weight", rotations[0]), (k, "k_weight", rotations[1])):
            x = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt()
            x = x * P[name] if m.qk_norm else x
            new.append(x if rotation is None else rotate(x, rotation))
        q, k = new
    w = torch.from_numpy(m.plan.quad_weights()).cuda().log().repeat_interleave(m.plan.nlon_in)
    s = q.flatten(2, 3) @ k.flatten(2, 3).transpose(2, 3) / m.head_dim ** 0.5 + w
    y = (torch.softmax(s, -1) @ v.flatten(2, 3)).unflatten(2, q.shape[2:4]).permute(0, 1, 4, 2, 3).flatten(1, 2)
    y = torch.nn.functional.conv2d(y, P["wo"], P["bo"])
    return y if residual is None else residual + y


def off(a, b):
    return float((a.detach().double() - b.detach()).norm() / b.detach().norm())


@pytest.mark.parametrize("options, bound", [
    # fp32 operators: 1e-4 of the largest value per gradient, and products in fp32 around them
    (dict(qk_norm=True), 1e-3), (dict(rotary=True), 1e-3), (dict(qk_norm=True, rotary=True), 1e-3),
    # queries and keys rounded to bfloat16 move a score by at most sqrt(C) 2^-8 = 0.022 for C = 32 (unit rows, scale 1 / sqrt(C)); v, p, ds and the result add 2^-9
    # each, and a gradient passes two such steps
    (dict(half_attention=True, qk_norm=True, rotary=True), 2 * (2 * 0.022 + 4 * 2.0 ** -9)), (dict(half_attention=True), 2 * (2 * 0.022 + 4 * 2.0 ** -9)),
], ids=lambda v: "-".join(v) if isinstance(v, dict) else "")
def test_a_training_step_against_64_bits(options, bound):
    torch.manual_seed(0)
    plan = sna.Plan(12, 24, 6, 12, 1, 1, global_attention=True)
    m = SphericalNeighborhoodAttention(plan, 20, 2, 32, **options).cuda()
    for p in m.parameters():
        p.data += 0.1 * torch.randn_like(p)
    x_q, x_kv, r = torch.randn(2, 20, 6, 12, device="cuda").requires_grad_(), torch.randn(2, 20, 12, 24, device="cuda").requires_grad_(), torch.randn(2, 20, 6, 12, device="cuda")
    y = m(x_q, x_kv, r)
    g = torch.randn_like(y)
    ends = [x_q, x_kv, *m.parameters()]
    grads = torch.autograd.grad(y, ends, g)
    doubles = [x_q.detach().double().requires_grad_(), x_kv.detach().double().requires_grad_()]
    ref = plain(m, *doubles, r.double())
    refs = torch.autograd.grad(ref, doubles + list(m.parameters()), g.double())
    assert off(y, ref) < bound
    largest = max(float(b.double().norm()) for b in refs)
    for (name, _), a, b in zip([("x_q", 0), ("x_kv", 0), *m.named_parameters()], grads, refs):
        # (the gradient of bk is zero without a rotation: a shift of all keys changes nothing)
        assert float((a.double() - b.double()).norm()) <= bound * max(float(b.double().norm()), 1e-2 * largest), name


def test_off_by_default_and_what_ran_before_is_the_same():
    torch.manual_seed(1)
    plan = sna.Plan(12, 24, 12, 24, 0, 0, 0.6)
    m = SphericalNeighborhoodAttention(plan, 8, 2, 16).cuda()
    assert sorted(n for n, _ in m.named_parameters()) == ["bk", "bo", "bq", "bv", "wk", "wo", "wq", "wv"] and not list(m.buffers())
    x = torch.randn(1, 8, 12, 24, device="cuda")
    y = m(x)
    assert torch.equal(m(x, residual=x), x + y) and torch.equal(m.train()(x), y)


def test_neighborhoods_with_norm_and_rotation():
    """A cutoff: the fp32 operator on what the norm and the rotation give."""
    torch.manual_seed(2)
    plan = sna.Plan(16, 32, 8, 16, 0, 0, 0.9)
    m = SphericalNeighborhoodAttention(plan, 8, 2, 16, qk_norm=True, rotary=True).cuda()
    x_q, x_kv = torch.randn(2, 8, 8, 16, device="cuda"), torch.randn(2, 8, 16, 32, device="cuda")
    y = m(x_q, x_kv)
    conv = torch.nn.functional.conv2d
    q, k, v = (conv(x.contiguous(memory_format=torch.channels_last), w, b).unflatten(1, (2, 16)).permute(0, 1, 3, 4, 2)
               for x, w, b in ((x_q, m.wq, m.bq), (x_kv, m.wk, m.bk), (x_kv, m.wv, m.bv)))
    q, k = layer.qk_norm_rotate(q, k, m.q_weight, m.k_weight, *layer.plan_rotations(plan, 16))
    ref = conv(plan.forward(q.detach().contiguous(), k.detach().contiguous(), v.detach().contiguous()).permute(0, 1, 4, 2, 3).flatten(1, 2), m.wo, m.bo)
    assert float((y - ref).abs().max()) <= 1e-5 * float(ref.abs().max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_module_of_16_bits(dtype):
    torch.manual_seed(3)
    plan = sna.Plan(12, 24, 12, 24, 1, 1, global_attention=True)
    m = SphericalNeighborhoodAttention(plan, 16, 2, 32, half_attention=True, qk_norm=True, rotary=True, dropout=0.25).cuda().to(dtype)
    x = torch.randn(2, 16, 12, 24, device="cuda", dtype=dtype).requires_grad_()
    y = m(x, residual=x)
    assert y.dtype == dtype and y.shape == x.shape
    y.float().square().sum().backward()
    assert all(p.grad is not None and bool(torch.isfinite(p.grad).all()) and p.grad.dtype == dtype for p in m.parameters())
    share = float((y == x).double().mean())
    assert abs(share - 0.25) < 5 * math.sqrt(0.25 * 0.75 / y.numel()) + 2e-2      # (a kept value may be too small to show)
    m.eval()
    assert torch.equal(m(x), m(x))


def test_dropout_under_checkpointing_and_copies():
    torch.manual_seed(4)
    plan = sna.Plan(12, 24, 12, 24, 1, 1, global_attention=True)
    m = SphericalNeighborhoodAttention(plan, 16, 2, 32, half_attention=True, qk_norm=True, dropout=0.5).cuda()
    x = torch.randn(2, 16, 12, 24, device="cuda").requires_grad_()
    torch.manual_seed(7)
    y = m(x, residual=x)
    ref = torch.autograd.grad(y.square().sum(), x)[0]
    torch.manual_seed(7)
    z = torch.utils.checkpoint.checkpoint(lambda t: m(t, residual=t), x, use_reentrant=False)
    assert torch.equal(y, z) and torch.equal(torch.autograd.grad(z.square().sum(), x)[0], ref)
    twin = copy.deepcopy(m)
    torch.manual_seed(7)
    assert torch.equal(twin(x, residual=x), y)


def test_a_captured_training_step():
    torch.manual_seed(5)
    plan = sna.Plan(12, 24, 12, 24, 1, 1, global_attention=True)
    m = SphericalNeighborhoodAttention(plan, 16, 2, 32, half_attention=True, qk_norm=True, rotary=True).cuda()
    x = torch.randn(2, 16, 12, 24, device="cuda")
    params = list(m.parameters())

    def step():
        y = m(x, residual=x)
        return tuple(t.detach() for t in (y, *torch.autograd.grad(y.square().sum(), params)))

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(3):
            step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    x.copy_(torch.randn_like(x))
    graph.replay()
    for a, b in zip(step(), captured):
        assert float((a.double() - b.double()).norm()) <= 1e-5 * float(b.double().norm())       # (the library's products may choose another kernel)


def test_refusals():
    plan = sna.Plan(12, 24, 12, 24, 0, 0, 0.6)
    with pytest.raises(ValueError, match="global plan"):
        SphericalNeighborhoodAttention(plan, 8, 2, 16, half_attention=True)
    full = sna.Plan(12, 24, 12, 24, 0, 0, global_attention=True)
    with pytest.raises(ValueError, match="multiple of 8"):
        SphericalNeighborhoodAttention(full, 8, 2, 12, half_attention=True)
    with pytest.raises(ValueError, match="dropout"):
        SphericalNeighborhoodAttention(full, 8, 2, 16, dropout=1.0)


def test_training_after_a_first_call_in_inference_mode():
    torch.manual_seed(6)
    plan = sna.Plan(6, 12, 6, 12, 0, 0, global_attention=True)
    m = SphericalNeighborhoodAttention(plan, 8, 2, 16, qk_norm=True, rotary=True, half_attention=True).cuda()
    x = torch.randn(2, 8, 6, 12, device="cuda")
    with torch.inference_mode():
        first = m(x)
    y = m(x)
    y.sum().backward()
    assert torch.equal(first, y) and all(bool(torch.isfinite(p.grad).all()) for p in m.parameters())


@pytest.mark.parametrize("shape", [(2, 8, 12, 24), (1, 8, 1, 1)])
def test_residuals_of_another_type_or_shape_with_dropout(shape):
    torch.manual_seed(7)
    plan = sna.Plan(12, 24, 12, 24, 0, 0, global_attention=True)
    m = SphericalNeighborhoodAttention(plan, 8, 2, 16, half_attention=True, dropout=0.25).cuda()
    x, residual = torch.randn(2, 8, 12, 24, device="cuda"), torch.randn(*shape, device="cuda", requires_grad=True)
    with torch.autocast("cuda", torch.bfloat16):
        rest = m.eval()(x)
        kept = m.train()(x, residual=residual)
    assert rest.dtype == torch.bfloat16 and kept.dtype == torch.float32
    # a kept value of the attention's result in 16 bits, divided by 0.75 in 32 and added in one rounding; half a unit of the sum and of the quotient
    y = kept.detach().double() - residual.detach().double()
    quotient = rest.detach().double() / 0.75
    room = 2.0 ** -23 * (quotient.abs() + kept.detach().double().abs() + residual.detach().double().abs())
    dropped = y.abs() <= room
    assert bool((dropped | ((y - quotient).abs() <= room)).all()) and 0.2 < float(dropped.double().mean()) < 0.3
    kept.sum().backward()
    assert torch.equal(residual.grad, torch.full(shape, 2 * 8 * 12 * 24 / residual.numel(), device="cuda"))


def test_more_residuals_than_results_with_dropout():
    """One result and a batch of residuals, as the plain sum takes them: the result is dropped once."""
    torch.manual_seed(8)
    plan = sna.Plan(6, 12, 6, 12, 0, 0, global_attention=True)
    m = SphericalNeighborhoodAttention(plan, 8, 2, 16, half_attention=True, dropout=0.25).cuda()
    x, residual = torch.randn(1, 8, 6, 12, device="cuda"), torch.randn(3, 8, 6, 12, device="cuda", requires_grad=True)
    assert m.eval()(x, residual=residual).shape == residual.shape
    m.train()
    torch.manual_seed(9)
    kept = m(x, residual=residual)
    torch.manual_seed(9)
    assert torch.equal(kept, residual + m(x))
    kept.sum().backward()
    assert torch.equal(residual.grad, torch.ones_like(residual)) and bool(torch.isfinite(m.wo.grad).all())
    with pytest.raises(RuntimeError, match="broadcast|must match|not match"):
        m(x, residual=residual[:, :, :5])
