"""Multi-head spherical (neighborhood) attention as a ``torch.nn.Module`` on channels-first feature maps.

The paper's attention layer (Sec. 3.3, "spherical multi-head attention") projects a feature map to queries, keys and
values with pointwise (1x1) linear maps, splits the channels into heads, applies the attention operator and projects
the result back.  Only the attention operator is this package's subject: the four pointwise projections here are plain
``torch.nn.functional.conv2d`` calls (library GEMMs), and the operator is the channels-first entry point of the C ABI,
so no tensor is permuted in Python.

A layer of a transformer usually does more, and can here: normalise its queries and keys per head and rotate them by position, compute
global attention in 16 bits, drop values of its result and add the residual (layer.py).  All of that is off unless asked for.
"""
from __future__ import annotations

import math

import torch

from . import layer, sna
from .autograd import spherical_neighborhood_attention, spherical_neighborhood_attention_cf


class SphericalNeighborhoodAttention(torch.nn.Module):
    """x_q [B, C_in, nlat_out, nlon_out], x_kv [B, C_in, nlat_in, nlon_in] -> [B, C_out, nlat_out, nlon_out].

    ``plan`` fixes grids and cutoff (``sna.Plan(..., global_attention=True)`` gives global spherical attention).
    ``embed_dim`` = heads * head_dim channels are used inside; head_dim must be a multiple of 4 up to 128.

    ``qk_norm``: queries and keys are normalised over each head's channels, with a learned weight per channel (``layer.qk_norm_rotate``).
    ``rotary``: they are rotated by the position of their point, half of the pairs of channels by colatitude, half by longitude
    (``layer.plan_rotations``); implies the norm, whose weights stay ones without ``qk_norm``.
    ``half_attention``: attention of 16-bit queries, keys and values (the input's type if that has 16 bits, else bfloat16) by
    ``layer.weighted_attention``; needs a global plan and a head_dim that is a multiple of 8.
    ``dropout``: share of the result's values that training drops, without a stored mask (``layer.residual_dropout``; random numbers from
    PyTorch's generator of the device).  ``forward(..., residual=r)`` returns r plus the (dropped) result.

    Tables of angles and weights are made on the first call on a device: make it outside any stream capture.
    """

    def __init__(self, plan: "sna.Plan", in_channels: int, heads: int, head_dim: int, out_channels: int | None = None, bias: bool = True, *,
                 qk_norm: bool = False, rotary: bool = False, half_attention: bool = False, dropout: float = 0.0):
        super().__init__()
        if head_dim % 4 != 0 or not 4 <= head_dim <= 128:
            raise ValueError("head_dim must be a multiple of 4 between 4 and 128")
        if half_attention and (not plan.global_attention or head_dim % 8 != 0):
            raise ValueError("half_attention needs a global plan and a head_dim that is a multiple of 8")
        if not 0.0 <= dropout < 1.0:
            raise ValueError("dropout must be at least 0 and less than 1")
        self.qk_norm, self.rotary, self.half_attention, self.dropout = qk_norm, rotary, half_attention, dropout
        self.q_weight = torch.nn.Parameter(torch.ones(head_dim)) if qk_norm else None
        self.k_weight = torch.nn.Parameter(torch.ones(head_dim)) if qk_norm else None
        self._tables = {}        # per device: rotations of queries and keys, logarithmic weights
        self.plan, self.heads, self.head_dim = plan, heads, head_dim
        embed = heads * head_dim
        out_channels = in_channels if out_channels is None else out_channels
        make = lambda o, i: torch.nn.Parameter(torch.empty(o, i, 1, 1).uniform_(-1.0 / math.sqrt(i), 1.0 / math.sqrt(i)))
        self.wq, self.wk, self.wv, self.wo = make(embed, in_channels), make(embed, in_channels), make(embed, in_channels), make(out_channels, embed)
        self.bq = torch.nn.Parameter(torch.zeros(embed)) if bias else None
        self.bk = torch.nn.Parameter(torch.zeros(embed)) if bias else None
        self.bv = torch.nn.Parameter(torch.zeros(embed)) if bias else None
        self.bo = torch.nn.Parameter(torch.zeros(out_channels)) if bias else None

    def _tables_on(self, device):
        if device not in self._tables:
            with torch.inference_mode(False):       # (they outlive the first call, whose mode may not be the next one's)
                rotations = layer.plan_rotations(self.plan, self.head_dim, device) if self.rotary else (None, None)
                self._tables[device] = (*rotations, layer.log_quadrature_weights(self.plan, device) if self.half_attention else None)
        return self._tables[device]

    def _attend_by_heads(self, q, k, v):
        """Channels-first projections [B, heads * C, nlat, nlon] -> [B, heads * C, nlat, nlon], through [B, heads, nlat, nlon, C]."""
        q_rotation, k_rotation, log_weights = self._tables_on(q.device)
        split = lambda x: x.unflatten(1, (self.heads, self.head_dim)).permute(0, 1, 3, 4, 2)
        q, k, v = split(q), split(k), split(v)
        if self.qk_norm or self.rotary:
            # (the norm's weights and the tables are kept in fp32 whatever the module's type)
            weights = (self.q_weight.float(), self.k_weight.float()) if self.qk_norm else (None, None)
            q, k = layer.qk_norm_rotate(q, k, *weights, q_rotation, k_rotation)
        if self.half_attention:
            dtype = q.dtype if q.dtype in (torch.bfloat16, torch.float16) else torch.bfloat16
            y = layer.weighted_attention(q.to(dtype), k.to(dtype), v.to(dtype), log_weights)
        else:
            y = spherical_neighborhood_attention(self.plan, q.float(), k.float(), v.float())
        return y.permute(0, 1, 4, 2, 3).flatten(1, 2)

    def forward(self, x_q: torch.Tensor, x_kv: torch.Tensor | None = None, residual: torch.Tensor | None = None) -> torch.Tensor:
        x_kv = x_q if x_kv is None else x_kv
        conv = torch.nn.functional.conv2d
        by_heads = self.qk_norm or self.rotary or self.half_attention
        if by_heads:
            # with the channels innermost the projections leave them so, and the heads are read in place
            same = x_kv is x_q
            x_q = x_q.contiguous(memory_format=torch.channels_last)
            x_kv = x_q if same else x_kv.contiguous(memory_format=torch.channels_last)
        q = conv(x_q, self.wq, self.bq)          # channel h * head_dim + c is channel c of head h: the layout sna_forward_cf takes
        k = conv(x_kv, self.wk, self.bk)
        v = conv(x_kv, self.wv, self.bv)
        if by_heads:
            y = self._attend_by_heads(q, k, v)
        else:
            y = spherical_neighborhood_attention_cf(self.plan, q.float(), k.float(), v.float(), heads=self.heads)
        y = conv(y.to(x_q.dtype), self.wo, self.bo)
        if self.training and self.dropout > 0.0:
            if residual is not None:        # (of other types, under autocast say: as the plain sum takes them)
                dtype = torch.promote_types(y.dtype, residual.dtype)
                y, residual = y.to(dtype), residual.to(dtype)
                if torch.broadcast_shapes(y.shape, residual.shape) != y.shape:      # (several residuals of one result, dropped once)
                    return residual + layer.residual_dropout(y, layer.dropout_state(y.device), self.dropout)
                residual = residual.expand_as(y)
            return layer.residual_dropout(y, layer.dropout_state(y.device), self.dropout, residual)
        return y if residual is None else residual + y
