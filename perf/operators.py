"""Timing cases of the operators around the attention of a layer, and their plain forms.

Three operators, in the order in which an attention layer uses them:

* ``rotate``  - queries and keys normalised per head (root mean square over the channels, times a weight) and rotated by the
  position of their grid point, in one pass; and its gradient (queries, keys, both weights);
* ``attend``  - softmax attention of 16-bit queries over all points of a grid, with a logarithmic weight per point (quadrature
  weights; points of weight zero take no part), its gradient with recomputed probabilities, and its form for few queries;
* ``dropout`` - residual + dropout(x), random numbers from a counter-based generator (Philox 4x32, ten rounds) keyed by a seed
  and an offset that are inputs, the mask never stored; and its gradient.

A case holds plain values: ``op``, ``dtype``, ``train`` (forward and backward; otherwise forward only) and sizes: grids
``nlat_q x nlon_q`` of the queries and ``nlat_k x nlon_k`` of keys and values, batch ``B``, heads ``Hq`` and ``Hk`` (a key head
serves Hq / Hk query heads), ``C`` channels per head.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
EPS = 1e-6
EXCLUDED = -1e30      # a point whose logarithmic weight is not above this takes no part


def _rotate(name, q_grid, k_grid, B, Hq, Hk, C, dtype, train, pairs_lat, pairs_lon, interleaved=False, token_major=False):
    case = {"name": name, "op": "rotate", "dtype": dtype, "train": train, "nlat_q": q_grid[0], "nlon_q": q_grid[1],
            "nlat_k": k_grid[0], "nlon_k": k_grid[1], "B": B, "Hq": Hq, "Hk": Hk, "C": C, "pairs_lat": pairs_lat,
            "pairs_lon": pairs_lon, "interleaved": interleaved, "token_major": token_major}
    return {key: value for key, value in case.items() if value is not None}


def _attend(name, q_grid, k_grid, B, Hq, Hk, C, dtype, train, weights="grid", token_major=False):
    """weights: "none", "grid" (quadrature weights) or "masked" (also points left out, their keys and values NaN; the last batch
    has no point left when there are several)."""
    case = {"name": name, "op": "attend", "dtype": dtype, "train": train, "nlat_q": q_grid[0], "nlon_q": q_grid[1],
            "nlat_k": k_grid[0], "nlon_k": k_grid[1], "B": B, "Hq": Hq, "Hk": Hk, "C": C, "weights": weights,
            "token_major": token_major}
    return {key: value for key, value in case.items() if value is not None}


def _dropout(name, shape, dtype, train, p, residual=True):
    case = {"name": name, "op": "dropout", "dtype": dtype, "train": train, "B": shape[0], "points": shape[1],
            "channels": shape[2], "p": p, "residual": residual}
    return {key: value for key, value in case.items() if value is not None}


def listed():
    return [
        # the smallest call: one head on a coarse grid, forward only; latency
        _rotate("rotate_coarse_infer", (32, 64), (32, 64), 1, 1, 1, 16, "float32", False, 4, 4),
        # a training step's queries and keys on panoramas, embedding 128 in four heads
        _rotate("rotate_pano128_train", (128, 256), (128, 256), 4, 4, 4, 32, "float32", True, 8, 8),
        # a down-sampling layer in 16 bits: keys on the finer grid; the largest
        _rotate("rotate_down256_train", (128, 256), (256, 512), 2, 8, 8, 32, "bfloat16", True, 8, 8),
        # an odd grid, a ragged head width, shared key heads, tensors that a projection left with the points outermost
        _rotate("rotate_gauss91_infer", (91, 180), (91, 180), 2, 8, 2, 24, "float16", False, 5, 6, True, True),
        # queries at one station over whole fields of a Gaussian grid, shared key heads: a served request
        _attend("attend_station_infer", (1, 1), (361, 720), 2, 8, 2, 64, "bfloat16", False),
        # global attention of a coarse level, one field: a short call
        _attend("attend_coarse_infer", (32, 64), (32, 64), 1, 4, 4, 32, "bfloat16", False),
        # training step of a global layer
        _attend("attend_global64_train", (64, 128), (64, 128), 2, 4, 4, 32, "bfloat16", True),
        # wide heads, more of them: the largest
        _attend("attend_global64_c128_train", (64, 128), (64, 128), 2, 8, 8, 128, "bfloat16", True),
        # ocean fields: land points are left out (and hold NaN), one field is all land; odd grids, a head width that is no
        # power of two, shared key heads, points outermost
        _attend("attend_masked_train", (45, 90), (61, 121), 3, 6, 2, 40, "float16", True, "masked", True),
        # the smallest dropout: an output of one head on a coarse grid
        _dropout("dropout_coarse_train", (1, 32 * 64, 16), "float32", True, 0.1),
        # the residual of a layer with 256 channels on panoramas
        _dropout("dropout_pano128_train", (4, 128 * 256, 256), "bfloat16", True, 0.1),
        # an odd number of values, no residual
        _dropout("dropout_gauss91_train", (3, 91 * 181, 77), "float16", True, 0.25, False),
    ]


def _log_uniform(rng, low, high):
    return round(math.exp(rng.uniform(math.log(low), math.log(high))))


def draw(rng):
    """Grids of 1 to 361 rings (attention: up to 96 for fields, down to single points), heads of 8 to 128 channels."""
    op = rng.choice(["rotate", "attend", "attend", "attend", "dropout"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16"] + ([] if op == "attend" else ["float32"]))
    train = rng.random() < 0.6
    B = rng.choice([1, 1, 2, 3, 4])
    if op == "dropout":
        channels = rng.choice([1, 16, 32, 77, 96, 128, 255, 256])
        points = _log_uniform(rng, 1, 4 * 128 * 256 * 256 // (B * channels))
        return _dropout(None, (B, points, channels), dtype, train, rng.choice([0.0, 0.05, 0.1, 0.3, 0.5]), rng.random() < 0.7)
    Hk = rng.choice([1, 2, 3, 4, 8])
    Hq = Hk * rng.choice([1, 1, 1, 2, 4])
    token_major = rng.random() < 0.3
    if op == "rotate":
        C = rng.choice([4, 8, 16, 24, 32, 32, 64, 80, 128])
        largest = 2 * 8 * 32 * 5 * 128 * 256
        while True:
            nlat_q, nlat_k = _log_uniform(rng, 1, 361), _log_uniform(rng, 1, 361)
            grids = (nlat_q, max(1, 2 * nlat_q + rng.choice([-1, 0, 0, 3]))), (nlat_k, max(1, 2 * nlat_k + rng.choice([0, 0, 1])))
            if B * C * (Hq * grids[0][0] * grids[0][1] + Hk * grids[1][0] * grids[1][1]) <= largest:
                break
            Hq, Hk, B = max(1, Hq // 2), 1, max(1, B - 1)
        pairs = rng.choice([C // 2, C // 2, C // 4])
        pairs_lat = rng.choice([pairs // 2, pairs // 2, 0, pairs])
        return _rotate(None, *grids, B, Hq, Hk, C, dtype, train, pairs_lat, pairs - pairs_lat, rng.random() < 0.5, token_major)
    C = rng.choice([8, 16, 24, 32, 32, 40, 64, 64, 80, 96, 128])
    weights = rng.choice(["none", "grid", "grid", "masked"])
    if rng.random() < 0.25:       # few queries over many points
        nlat_k = _log_uniform(rng, 1, 361)
        return _attend(None, (1, rng.choice([1, 1, 2, 7, 16])), (nlat_k, max(1, 2 * nlat_k + rng.choice([-1, 0, 0]))), min(B, 2), Hq, Hk, min(C, 64),
                       dtype, False, weights, token_major)
    largest = 2 * 8 * 128 * (64 * 128) ** 2
    while True:
        nlat_q = _log_uniform(rng, 1, 96)
        nlat_k = rng.choice([nlat_q, nlat_q, _log_uniform(rng, 1, 96)])
        grids = (nlat_q, max(1, 2 * nlat_q + rng.choice([-1, 0, 0, 5]))), (nlat_k, max(1, 2 * nlat_k + rng.choice([0, 0, 1])))
        pairs = B * Hq * grids[0][0] * grids[0][1] * grids[1][0] * grids[1][1]
        if pairs * C <= largest and pairs <= 2e9:
            return _attend(None, *grids, B, Hq, Hk, C, dtype, train, weights, token_major)


def _angles(count, pairs, step):
    """count x pairs angles in 64 bits: whole multiples of a position's angle, from 1 upwards by powers of two and between."""
    waves = torch.tensor([float(max(1, round(1.5 ** p))) for p in range(pairs)], dtype=torch.float64)
    return torch.arange(count, dtype=torch.float64)[:, None] * step * waves[None, :]


def _table(count, pairs, step, device):
    angle = _angles(count, pairs, step)
    return torch.stack((angle.cos(), angle.sin()), -1).float().to(device)


def _heads(gen, B, H, nlat, nlon, C, dtype, token_major, scale=1.0):
    if token_major:
        x = scale * torch.randn(B, nlat, nlon, H, C, generator=gen, device="cuda")
        return x.to(dtype).permute(0, 3, 1, 2, 4)
    return (scale * torch.randn(B, H, nlat, nlon, C, generator=gen, device="cuda")).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype, B = DTYPES[case["dtype"]], case["B"]
    state = {"op": case["op"], "train": case["train"]}
    if case["op"] == "dropout":
        shape = (B, case["points"], case["channels"])
        state["x"] = torch.randn(shape, generator=gen, device="cuda").to(dtype)
        state["residual"] = torch.randn(shape, generator=gen, device="cuda").to(dtype) if case["residual"] else None
        state["rng"] = torch.randint(-2 ** 62, 2 ** 62, (2,), generator=gen, device="cuda", dtype=torch.int64)
        state["p"] = case["p"]
        state["dout"] = torch.randn(shape, generator=gen, device="cuda").to(dtype)
        leaves = ("x", "residual")
    else:
        Hq, Hk, C, outermost = case["Hq"], case["Hk"], case["C"], case["token_major"]
        q_grid, k_grid = (case["nlat_q"], case["nlon_q"]), (case["nlat_k"], case["nlon_k"])
        state["q"] = _heads(gen, B, Hq, *q_grid, C, dtype, outermost)
        state["k"] = _heads(gen, B, Hk, *k_grid, C, dtype, outermost)
        if case["op"] == "rotate":
            state["q_weight"] = 1 + 0.2 * torch.randn(C, generator=gen, device="cuda")
            state["k_weight"] = 1 + 0.2 * torch.randn(C, generator=gen, device="cuda")
            for name, (nlat, nlon) in (("q", q_grid), ("k", k_grid)):
                state[name + "_rotation"] = (_table(nlat, case["pairs_lat"], math.pi / max(1, nlat - 1), "cuda"),
                                             _table(nlon, case["pairs_lon"], 2 * math.pi / nlon, "cuda"))
            state["interleaved"] = case["interleaved"]
            state["dq"], state["dk"] = _heads(gen, B, Hq, *q_grid, C, dtype, outermost), _heads(gen, B, Hk, *k_grid, C, dtype, outermost)
            leaves = ("q", "k", "q_weight", "k_weight")
        else:
            state["v"] = _heads(gen, B, Hk, *k_grid, C, dtype, outermost)
            state["dout"] = _heads(gen, B, Hq, *q_grid, C, dtype, outermost)
            state["log_weights"] = None
            if case["weights"] != "none":
                ring = np.log(np.polynomial.legendre.leggauss(k_grid[0])[1] * 2 * math.pi / k_grid[1])
                state["log_weights"] = torch.from_numpy(ring).float().cuda().repeat_interleave(k_grid[1])
            if case["weights"] == "masked":
                patches = torch.rand(B, -(-k_grid[0] // 4), -(-k_grid[1] // 4), generator=gen, device="cuda") < 0.4
                land = patches.repeat_interleave(4, 1).repeat_interleave(4, 2)[:, :k_grid[0], :k_grid[1]]
                if B > 1:
                    land[-1] = True
                state["log_weights"] = state["log_weights"].masked_fill(land.reshape(B, -1), -math.inf)
                for name in "kv":
                    state[name].masked_fill_(land[:, None, :, :, None], math.nan)
            leaves = ("q", "k", "v")
    if case["train"]:
        for name in leaves:
            if state[name] is not None:
                state[name].requires_grad_(True)
    return state


# ---- the plain forms ------------------------------------------------------------------------------------------------------

def _rotation_of(rotation, forwards):
    """cos and sin of every pair at every grid point, [nlat, nlon, pairs]."""
    lat, lon = rotation
    shape = (lat.shape[0], lon.shape[0])
    both = torch.cat((lat[:, None].expand(*shape, -1, 2), lon[None].expand(*shape, -1, 2)), 2)
    return both[..., 0], both[..., 1] if forwards else -both[..., 1]


def _turn(x, rotation, interleaved, forwards=True):
    cos, sin = _rotation_of(rotation, forwards)
    pairs = cos.shape[-1]
    if interleaved:
        first, second = x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]
    else:
        first, second = x[..., :pairs], x[..., pairs:2 * pairs]
    a, b = first * cos - second * sin, first * sin + second * cos
    turned = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., 2 * pairs:]), -1)


def _plain_rotate(x, weight, rotation, interleaved, grad):
    x32 = x.detach().float()
    inverse = torch.rsqrt(x32.square().mean(-1, keepdim=True) + EPS)
    normal = x32 * inverse
    if grad is None:
        return _turn(normal * weight.detach(), rotation, interleaved).to(x.dtype)
    g = _turn(grad.float(), rotation, interleaved, forwards=False)
    dweight = (g * normal).sum((0, 1, 2, 3))
    g = g * weight.detach()
    return (inverse * (g - normal * (g * normal).mean(-1, keepdim=True))).to(x.dtype), dweight


def _plain_attend(state):
    q, k, v = (state[name].detach().float().flatten(2, 3) for name in "qkv")
    B, Hq, Nq, C = q.shape
    Hk, Nk = k.shape[1:3]
    scale = 1 / math.sqrt(C)
    rows = lambda x: x.reshape(B, Hk, Hq // Hk * Nq, C)      # the query heads that share a key head, one below the other
    bias = torch.zeros(1, 1, 1, Nk, device=q.device) if state["log_weights"] is None else state["log_weights"].reshape(-1, 1, 1, Nk)
    left_out = bias <= EXCLUDED
    k, v = (torch.where(left_out.transpose(2, 3), 0.0, x) for x in (k, v))
    s = torch.where(left_out, -math.inf, rows(q) @ k.transpose(2, 3) * scale + bias)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    shape, dtype = state["q"].shape, state["q"].dtype
    out = (p @ v).reshape(shape).to(dtype)
    if not state["train"]:
        return out, (top + torch.log(total)).reshape(shape[:-1])
    dout = rows(state["dout"].float().flatten(2, 3))
    dv = p.transpose(2, 3) @ dout
    ds = dout @ v.transpose(2, 3)
    ds = p * (ds - (p * ds).sum(-1, keepdim=True)) * scale
    return (out, (ds @ k).reshape(shape).to(dtype), (ds.transpose(2, 3) @ rows(q)).reshape(state["k"].shape).to(dtype),
            dv.reshape(state["k"].shape).to(dtype))


def _philox(count, rng):
    """`count` blocks of four random 32-bit numbers: counter (block, offset), key the seed; all words in 64-bit integers."""
    low = 0xffffffff
    block = torch.arange(count, dtype=torch.int64, device=rng.device)
    key = [rng[0] & low, (rng[0] >> 32) & low]
    word = [block & low, block >> 32, (rng[1] & low).expand(count), ((rng[1] >> 32) & low).expand(count)]
    high_half = lambda a, b: ((b >> 16) * a + (((b & 0xffff) * a) >> 16)) >> 16
    for _ in range(10):
        word = [high_half(0xCD9E8D57, word[2]) ^ word[1] ^ key[0], (word[2] * 0xCD9E8D57) & low,
                high_half(0xD2511F53, word[0]) ^ word[3] ^ key[1], (word[0] * 0xD2511F53) & low]
        key = [(key[0] + 0x9E3779B9) & low, (key[1] + 0xBB67AE85) & low]
    return torch.stack(word, -1)


def _kept(x, p, rng):
    n = x.numel()
    return (_philox(-(-n // 4), rng).flatten()[:n] >= min(2 ** 32 - 1, round(p * 2 ** 32))).reshape(x.shape)


def _plain_dropout(state):
    x, residual, scale = state["x"].detach(), state["residual"], 1 / (1 - state["p"])
    kept = _kept(x, state["p"], state["rng"])
    out = torch.where(kept, x.float() * scale, 0.0)
    out = (out if residual is None else out + residual.detach().float()).to(x.dtype)
    if not state["train"]:
        return out
    dx = torch.where(kept, state["dout"].float() * scale, 0.0).to(x.dtype)
    return (out, dx) if residual is None else (out, dx, state["dout"])


def run(state):
    if own:
        return _run_own(state)
    if state["op"] == "dropout":
        return _plain_dropout(state)
    if state["op"] == "attend":
        return _plain_attend(state)
    both = [(state[x], state[x + "_weight"], state[x + "_rotation"], state["interleaved"]) for x in "qk"]
    out = tuple(_plain_rotate(*args, None) for args in both)
    if not state["train"]:
        return out
    (dq, dq_weight), (dk, dk_weight) = (_plain_rotate(*args, grad) for args, grad in zip(both, (state["dq"], state["dk"])))
    return (*out, dq, dk, dq_weight, dk_weight)


def _run_own(state):
    from paper_2505_11157_b200 import layer
    if state["op"] == "dropout":
        x, residual = state["x"], state["residual"]
        out = layer.residual_dropout(x, state["rng"], state["p"], residual=residual)
        if not state["train"]:
            return out
        return (out, *torch.autograd.grad(out, (x,) if residual is None else (x, residual), state["dout"]))
    if state["op"] == "attend":
        q, k, v = state["q"], state["k"], state["v"]
        if not state["train"]:
            return layer.weighted_attention(q, k, v, log_weights=state["log_weights"], return_lse=True)
        out = layer.weighted_attention(q, k, v, log_weights=state["log_weights"])
        return (out, *torch.autograd.grad(out, (q, k, v), state["dout"]))
    q, k, q_weight, k_weight = state["q"], state["k"], state["q_weight"], state["k_weight"]
    out = layer.qk_norm_rotate(q, k, q_weight, k_weight, q_rotation=state["q_rotation"], k_rotation=state["k_rotation"],
                               eps=EPS, interleaved=state["interleaved"])
    if not state["train"]:
        return out
    return (*out, *torch.autograd.grad(out, (q, k, q_weight, k_weight), (state["dq"], state["dk"])))


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------

def work(case):
    size, B = (4 if case["dtype"] == "float32" else 2), case["B"]
    if case["op"] == "dropout":
        n = B * case["points"] * case["channels"]
        tensors = (3 if case["residual"] else 2) + (2 if case["train"] else 0)      # x, residual, out; dout, dx (the residual's gradient is dout)
        return {"bytes": tensors * n * size + 16, "flops": 2.0 * n * (2 if case["train"] else 1)}
    of_q, of_k = (case["nlat_" + x] * case["nlon_" + x] * B * case["C"] * case["H" + x] for x in "qk")
    if case["op"] == "rotate":
        # forward: read and written; backward: the input, the gradient, its own gradient
        tables = 8 * (case["pairs_lat"] * (case["nlat_q"] + case["nlat_k"]) + case["pairs_lon"] * (case["nlon_q"] + case["nlon_k"]))
        return {"bytes": (of_q + of_k) * size * (5 if case["train"] else 2) + tables, "flops": (of_q + of_k) * (20.0 if case["train"] else 7.0)}
    Nk = case["nlat_k"] * case["nlon_k"]
    present = 1.0 if case["weights"] != "masked" else 0.6 * (B - 1) / B if B > 1 else 0.6
    pairs = case["nlat_q"] * case["nlon_q"] * case["Hq"] * B * Nk * present
    weights = 0 if case["weights"] == "none" else 4 * Nk * (B if case["weights"] == "masked" else 1)
    if not case["train"]:
        return {"bytes": size * (2 * of_q + 2 * of_k * present) + weights, "flops": 4.0 * pairs * case["C"]}
    # forward q, out; k, v.  backward q, out, dout, dq; k, v, dk, dv
    return {"bytes": size * (6 * of_q + (4 * present + 2) * of_k) + weights, "flops": 14.0 * pairs * case["C"]}


# ---- the definitions, in 64 bits ------------------------------------------------------------------------------------------

def _exact_rotate(state):
    ends = [state[name].detach().double().requires_grad_() for name in ("q", "k", "q_weight", "k_weight")]
    out = []
    for x, weight, (lat, lon) in zip(ends[:2], ends[2:], (state["q_rotation"], state["k_rotation"])):
        # a pair as a complex number, times the unit number of its angle
        lat, lon = (torch.view_as_complex(t.double()) for t in (lat, lon))
        nlat, nlon, pairs = lat.shape[0], lon.shape[0], lat.shape[1] + lon.shape[1]
        unit = torch.cat((lat.unsqueeze(1).repeat(1, nlon, 1), lon.unsqueeze(0).repeat(nlat, 1, 1)), -1)
        y = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * weight
        pair = y[..., :2 * pairs].unflatten(-1, (pairs, 2) if state["interleaved"] else (2, pairs))
        pair = pair if state["interleaved"] else pair.transpose(-1, -2)
        pair = torch.view_as_real(torch.complex(pair[..., 0].contiguous(), pair[..., 1].contiguous()) * unit)
        pair = pair if state["interleaved"] else pair.transpose(-1, -2)
        out.append(torch.cat((pair.flatten(-2), y[..., 2 * pairs:]), -1))
    if not state["train"]:
        return tuple(y.detach() for y in out)
    return (*(y.detach() for y in out), *torch.autograd.grad(out, ends, (state["dq"].double(), state["dk"].double())))


def _exact_attend(state):
    q, k, v = (state[name].detach() for name in "qkv")
    B, Hq = q.shape[:2]
    Hk, C = k.shape[1], k.shape[4]
    results = [torch.zeros(x.shape, dtype=torch.float64, device=q.device) for x in (q, q, k, k)]
    statistic = torch.zeros(q.shape[:4], dtype=torch.float64, device=q.device)
    for b in range(B):
        weights = torch.ones(k.shape[2] * k.shape[3], dtype=torch.float64, device=q.device)
        if state["log_weights"] is not None:
            mine = state["log_weights"].reshape(-1, weights.numel())
            mine = mine[b % mine.shape[0]].double()
            weights = torch.where(mine > EXCLUDED, mine.exp(), 0.0)
        part = weights.nonzero().flatten()
        for h in range(Hq):
            g = h // (Hq // Hk)
            if part.numel() == 0:
                statistic[b, h] = -math.inf
                continue
            # only the points that take part
            ends = [q[b, h].reshape(-1, C).double().requires_grad_(state["train"]),
                    *(x[b, g].reshape(-1, C)[part].double().requires_grad_(state["train"]) for x in (k, v))]
            logits = torch.einsum("ic,jc->ij", ends[0], ends[1]) / C ** 0.5 + weights[part].log()
            out = torch.softmax(logits, 1) @ ends[2]
            results[0][b, h] = out.detach().reshape(q.shape[2:])
            if not state["train"]:
                statistic[b, h] = torch.logsumexp(logits, 1).reshape(q.shape[2:4])
                continue
            grads = torch.autograd.grad(out, ends, state["dout"][b, h].reshape(-1, C).double())
            results[1][b, h] = grads[0].reshape(q.shape[2:])
            for result, grad in zip(results[2:], grads[1:]):
                flat = torch.zeros(weights.numel(), C, dtype=torch.float64, device=q.device)
                flat[part] = grad
                result[b, g] += flat.reshape(k.shape[2:])
            del logits, out, grads, ends
    return tuple(results) if state["train"] else (results[0], statistic)


def _exact_dropout(state):
    # Philox by whole numbers of 64 bits on the host
    seed, offset = (int(x) & (2 ** 64 - 1) for x in state["rng"].tolist())
    x = state["x"].detach()
    n, mask = x.numel(), np.uint64(0xffffffff)
    c = [np.arange(-(-n // 4), dtype=np.uint64)]
    c = [c[0] & mask, c[0] >> np.uint64(32), np.full_like(c[0], offset & 0xffffffff), np.full_like(c[0], offset >> 32)]
    k0, k1 = seed & 0xffffffff, seed >> 32
    for _ in range(10):
        first, second = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(second >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), second & mask, (first >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), first & mask]
        k0, k1 = (k0 + 0x9E3779B9) & 0xffffffff, (k1 + 0xBB67AE85) & 0xffffffff
    kept = np.stack(c, 1).reshape(-1)[:n] >= np.uint64(min(2 ** 32 - 1, round(state["p"] * 2 ** 32)))
    factor = torch.from_numpy(kept).to(x.device).reshape(x.shape).double() / (1 - state["p"])
    out = factor * x.double() + (0.0 if state["residual"] is None else state["residual"].detach().double())
    if not state["train"]:
        return out
    dx = factor * state["dout"].double()
    return (out, dx) if state["residual"] is None else (out, dx, state["dout"].double())


def exact(case, seed):
    state = prepare(case, seed)
    return {"rotate": _exact_rotate, "attend": _exact_attend, "dropout": _exact_dropout}[state["op"]](state)
