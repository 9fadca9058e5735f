"""The operators around the attention of a layer, differentiable: what its queries and keys pass through, and its residual.

Nothing is computed here: the calls go to native autograd functions (csrc_torch/sna_layer.cpp) over the C ABI.  Tensors of grids are
[B, H, nlat, nlon, C] (heads leading, as everywhere in this package) with any strides over contiguous channels: a packed projection, or
one that left the channels last, is read in place.  Every call takes its tensors' device and that device's current stream; gradients are
computed once (``create_graph`` is refused, and so are tensors with a tangent of forward-mode differentiation), in a fixed order of sums: the
same call gives the same bits.
"""
from __future__ import annotations

import math

import torch

from . import sna
from .autograd import _sna_torch

_PLAIN = frozenset((torch.Tensor, torch.nn.Parameter, type(None)))


def _check_plain(*tensors):
    for t in tensors:
        if type(t) not in _PLAIN:
            raise ValueError(f"expected a plain torch.Tensor, got {type(t).__name__}")
    if torch._C._get_tracing_state() is not None:
        raise RuntimeError("this operator cannot be traced: the kernels are launched outside PyTorch's dispatcher")


def rotation_tables(nlat: int, nlon: int, lat_angles, lon_waves, device="cuda"):
    """(lat_table, lon_table) of a grid for :func:`qk_norm_rotate`, computed in 64 bits.

    ``lat_angles`` [nlat, pairs]: the angle of every pair at every ring, in radians (colatitude times a frequency, say).
    ``lon_waves``: one whole number of turns per circle of latitude and pair, so that scores do not see where longitude begins."""
    lat = torch.as_tensor(lat_angles, dtype=torch.float64).reshape(nlat, -1)
    waves = torch.as_tensor(lon_waves, dtype=torch.int64).reshape(-1)
    # m * j modulo nlon in whole numbers: the angle stays below a turn however large m is
    lon = torch.remainder(torch.arange(nlon, dtype=torch.int64)[:, None] * torch.remainder(waves, nlon)[None, :], nlon).double() * (2 * math.pi / nlon)
    return tuple(torch.stack((a.cos(), a.sin()), -1).float().contiguous().to(device) for a in (lat, lon))


def plan_rotations(plan: "sna.Plan", head_dim: int, device="cuda"):
    """Tables for the queries (output grid) and the keys (input grid) of a plan: half of the pairs of channels turn with the colatitude,
    half with the longitude, with 1, 2, 3, 4, 6, 8, 11, ... (sqrt 2 apart) turns per circle; at most half as many as the coarser grid has points."""
    pairs = head_dim // 2
    lat_pairs = pairs // 2
    top = max(1, min(plan.nlon_in, plan.nlon_out) // 2)
    waves = [min(top, max(p + 1 if p < 4 else 0, round(2 ** (p / 2)))) for p in range(pairs - lat_pairs)]
    theta_in, theta_out = (torch.from_numpy(t) for t in plan.colatitudes())
    frequencies = torch.tensor(waves[:lat_pairs], dtype=torch.float64)
    return (rotation_tables(plan.nlat_out, plan.nlon_out, theta_out[:, None] * frequencies, waves, device),
            rotation_tables(plan.nlat_in, plan.nlon_in, theta_in[:, None] * frequencies, waves, device))


def qk_norm_rotate(q, k, q_weight=None, k_weight=None, q_rotation=None, k_rotation=None, eps: float = 1e-6, interleaved: bool = False):
    """Queries and keys normalised over each head's channels (x / sqrt(mean(x^2) + eps) * weight) and rotated by position; one pass over both.

    q [B, Hq, nlat, nlon, C], k [B, Hk, nlat', nlon', C], float32, bfloat16 or float16, C a multiple of 4 up to 128; their grids and
    heads may differ.  ``*_weight``: float32 [C], or None for ones.  ``*_rotation``: a pair (lat_table [nlat, pairs_lat, 2], lon_table
    [nlon, pairs_lon, 2]) of cos and sin (:func:`rotation_tables`), or None for no rotation; pairs are the channels (2p, 2p + 1) if
    ``interleaved``, else (p, p + pairs).  ``eps`` may be zero for vectors that are not.  Differentiable in q, k and the weights."""
    q_lat, q_lon = (None, None) if q_rotation is None else q_rotation
    k_lat, k_lon = (None, None) if k_rotation is None else k_rotation
    _check_plain(q, k, q_weight, k_weight, q_lat, q_lon, k_lat, k_lon)
    return _sna_torch.qk_norm_rotate(q, k, q_weight, k_weight, q_lat, q_lon, k_lat, k_lon, eps, interleaved)


def weighted_attention(q, k, v, log_weights=None, scale: float | None = None, return_lse: bool = False):
    """Softmax attention of 16-bit tensors over all points of a grid: out_i = sum_j p_ij v_j, p_ij ~ exp(scale q_i.k_j + log_weights_j).

    q [B, Hq, nlat, nlon, C], k and v [B, Hk, nlat', nlon', C], bfloat16 or float16, C a multiple of 8 up to 128, Hq a multiple of Hk:
    query head h reads key head h // (Hq // Hk).  ``log_weights``: float32, [nlat' * nlon'] or one such row per batch; with the logarithms of
    quadrature weights (:func:`log_quadrature_weights`) this is global spherical attention.  A point at -1e30 or below (-inf, the lowest number of any
    type) is left out, whatever k and v hold there (others must be below 1e30); a row without points gives zeros, and no gradient, whatever q holds.  ``scale``: 1 / sqrt(C) if None.
    Returns out, or with ``return_lse`` (out, lse): the logarithm of each row's sum, float32 [B, Hq, nlat, nlon], not differentiable.
    Differentiable in q, k and v: what is kept for the backward pass is lse, and out with what its rounding took (a second tensor of out's size); the probabilities are
    recomputed, and all three gradients computed, also where one is wanted.  The backward pass is slow for up to 16 queries, or less than 64 points, against very many of
    the other: it walks those without cutting them."""
    _check_plain(q, k, v, log_weights)
    if scale is None:
        scale = q.shape[-1] ** -0.5 if q.dim() and q.shape[-1] else 1.0
    out, lse = _sna_torch.weighted_attention(q, k, v, log_weights, scale)
    return (out, lse) if return_lse else out


def log_quadrature_weights(plan: "sna.Plan", device="cuda") -> torch.Tensor:
    """The logarithm of the quadrature weight of every point of a plan's input grid, float32 [nlat_in * nlon_in] (-inf for weight zero)."""
    weights = torch.from_numpy(plan.quad_weights())
    return weights.log().float().repeat_interleave(plan.nlon_in).to(device)


def residual_dropout(x, state, p: float, residual=None):
    """residual + dropout(x): each value of x is kept with probability 1 - p and then divided by it, else dropped; no mask is stored.

    ``state``: int64 CUDA tensor (seed, offset) that the random numbers are computed from (:func:`dropout_state` draws one); it is kept
    for the backward pass, which draws the same numbers again, so it must not change until then.  ``residual``: of x's shape and type, or
    None.  0 <= p < 1.  float32, bfloat16 or float16; x and residual are taken in row-major order.  Differentiable in x and residual."""
    _check_plain(x, state, residual)
    return _sna_torch.residual_dropout(x, state, p, residual)


def dropout_state(device) -> torch.Tensor:
    """A new (seed, offset) from PyTorch's generator of the device: repeatable by ``torch.manual_seed``, kept by checkpointing, and drawn
    anew by every replay of a captured graph."""
    return torch.randint(-2 ** 63, 2 ** 63 - 1, (2,), dtype=torch.int64, device=device)
