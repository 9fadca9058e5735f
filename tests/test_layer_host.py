"""Host side of the layer's operators: refusals of the C ABI (nothing is launched), the generator's definition, angles."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2505_11157_b200 import layer, sna

lib = sna._lib


def philox(blocks, seed, offset, first=0):
    """[blocks, 4] words: Philox 4x32, ten rounds, counter (block, offset), key seed."""
    mask = np.uint64(0xffffffff)
    seed, offset = seed % 2 ** 64, offset % 2 ** 64
    index = np.arange(first, first + blocks, dtype=np.uint64)
    c = [index & mask, index >> np.uint64(32), np.full_like(index, offset & 0xffffffff), np.full_like(index, offset >> 32)]
    key = [seed & 0xffffffff, seed >> 32]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(key[0]), b & mask, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(key[1]), a & mask]
        key = [(key[0] + 0x9E3779B9) & 0xffffffff, (key[1] + 0xBB67AE85) & 0xffffffff]
    return np.stack(c, 1)


def test_known_answers_of_the_generator():
    # two of the vectors published with the generator (counter words, key words, result)
    assert philox(1, 0, 0)[0].tolist() == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert philox(1, 0x299f31d0a4093822, 0x0370734413198a2e, first=0x85a308d3243f6a88)[0].tolist() == [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]


def test_angles_are_exact_multiples():
    lat, lon = layer.rotation_tables(3, 720, [[0.5], [1.0], [1.5]], [1, 359, 10 ** 12 + 1], device="cpu")
    assert lat.shape == (3, 1, 2) and lon.shape == (720, 3, 2) and lat.dtype == lon.dtype == torch.float32
    for j in (0, 1, 359, 719):
        for p, m in enumerate((1, 359, 10 ** 12 + 1)):
            angle = 2 * math.pi * ((m * j) % 720) / 720
            assert lon[j, p].tolist() == [np.float32(math.cos(angle)), np.float32(math.sin(angle))]
    assert lat[2, 0].tolist() == [np.float32(math.cos(1.5)), np.float32(math.sin(1.5))]


def test_plan_rotations_fit_any_head():
    plan = sna.Plan(9, 16, 5, 8, 0, 0, 1.5, host_only=True)
    for C in (4, 8, 12, 32, 64, 128):
        out, inp = layer.plan_rotations(plan, C, device="cpu")
        assert out[0].shape[:2] == (5, C // 2 // 2) and inp[1].shape[:2] == (16, C // 2 - C // 2 // 2)


def part(**kw):
    t = sna.SnaTensor(4096, 8, 8, 8, 8)
    r = sna.SnaRotate(nlat=2, nlon=2, H=1, x=t, y=t, dy=t, dx=t)
    for name, value in kw.items():
        setattr(r, name, value)
    return r


def rotate(parts, dtype=0, B=1, C=8, eps=1e-6, backward=False, workspace=None, workspace_bytes=0):
    array = (sna.SnaRotate * max(1, len(parts)))(*parts)
    if backward:
        return lib.sna_norm_rotate_backward(array, len(parts), dtype, B, C, eps, 0, workspace, workspace_bytes, None)
    return lib.sna_norm_rotate_forward(array, len(parts), dtype, B, C, eps, 0, None)


@pytest.mark.parametrize("status, call", [
    (1, lambda: lib.sna_norm_rotate_forward(None, 1, 0, 1, 8, 1e-6, 0, None)),
    (1, lambda: rotate([])),
    (1, lambda: rotate([part()] * 3)),
    (1, lambda: rotate([part()], dtype=3)),
    (1, lambda: rotate([part()], B=-1)),
    (2, lambda: rotate([part()], C=6)),
    (2, lambda: rotate([part()], C=132)),
    (1, lambda: rotate([part()], eps=-1.0)),
    (1, lambda: rotate([part()], eps=math.nan)),
    (1, lambda: rotate([part(nlat=-1)])),
    (2, lambda: rotate([part(nlat=1 << 16, nlon=1 << 16)])),
    (1, lambda: rotate([part(pairs_lat=3, pairs_lon=2)])),
    (1, lambda: rotate([part(pairs_lat=2 ** 31 - 1, pairs_lon=2 ** 31 - 1)])),
    (1, lambda: rotate([part(pairs_lat=2)])),
    (1, lambda: rotate([part(pairs_lat=2, lat_table=4100)])),
    (1, lambda: rotate([part(weight=4098)])),
    (1, lambda: rotate([part(x=sna.SnaTensor(None, 8, 8, 8, 8))])),
    (1, lambda: rotate([part(y=sna.SnaTensor(4104, 8, 8, 8, 8))])),
    (1, lambda: rotate([part(y=sna.SnaTensor(4096, 8, 8, 8, 6))])),
    (1, lambda: rotate([part(), part(dx=sna.SnaTensor(4096, 2, 8, 8, 8))], backward=True)),
    (1, lambda: rotate([part(dweight=4096)], backward=True)),
    (7, lambda: rotate([part(dweight=4096)], backward=True, workspace=4096, workspace_bytes=lib.sna_norm_rotate_workspace_bytes(8) - 1)),
    (1, lambda: lib.sna_dropout(4096, None, 4096, 3, 8, 0.1, 4096, None)),
    (1, lambda: lib.sna_dropout(4096, None, 4096, 0, 8, 1.0, 4096, None)),
    (1, lambda: lib.sna_dropout(4096, None, 4096, 0, 8, math.nan, 4096, None)),
    (1, lambda: lib.sna_dropout(4096, None, 4096, 0, -1, 0.1, 4096, None)),
    (2, lambda: lib.sna_dropout(4096, None, 4096, 0, 1 << 39, 0.1, 4096, None)),
    (1, lambda: lib.sna_dropout(None, None, 4096, 0, 8, 0.1, 4096, None)),
    (1, lambda: lib.sna_dropout(4098, None, 4096, 0, 8, 0.1, 4096, None)),
    (1, lambda: lib.sna_dropout(4096, None, 4096, 0, 8, 0.1, 4100, None)),
    (0, lambda: lib.sna_dropout(None, None, None, 0, 0, 0.1, None, None)),
], ids=lambda v: None)
def test_the_c_abi_refuses(status, call):
    assert call() == status
    assert status == 0 or lib.sna_last_error_message() != b""


def attention(**kw):
    t = sna.SnaTensor(4096, 8, 8, 32, 8)
    a = sna.SnaAttention(B=1, Hq=2, Hk=1, C=8, nlat_q=2, nlon_q=4, nlat_k=2, nlon_k=4, q=t, k=t, v=t, out=t, dout=t, dq=t, dk=t, dv=t, lse=4096, scale=0.3)
    for name, value in kw.items():
        setattr(a, name, value)
    return a


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("status, a, dtype", [
    (2, attention(), 0), (2, attention(), 3), (2, attention(C=12), 1), (2, attention(C=136), 1), (1, attention(Hq=3, Hk=2), 1), (1, attention(Hq=3, Hk=0), 1),
    (1, attention(B=-1), 1), (1, attention(nlat_k=-1), 1), (1, attention(scale=math.inf), 1), (1, attention(scale=math.nan), 1),
    (2, attention(nlat_q=1 << 15, nlon_q=1 << 15), 1), (2, attention(B=1 << 30, Hq=1 << 4, Hk=1), 1), (1, attention(lse=4098), 1), (1, attention(log_weights=4098), 1),
    (1, attention(q=sna.SnaTensor(4104, 8, 8, 32, 8)), 1), (1, attention(k=sna.SnaTensor(4096, 8, 8, 32, 4)), 1), (1, attention(v=sna.SnaTensor(4096, 8, 8, 40, 8)), 2),
    (1, attention(out=sna.SnaTensor(None, 8, 8, 32, 8)), 2),
], ids=lambda v: None)
def test_the_c_abi_refuses_attention(status, a, dtype, backward):
    call, size = (lib.sna_attention_backward, lib.sna_attention_backward_workspace_bytes) if backward else (lib.sna_attention_forward, lib.sna_attention_forward_workspace_bytes)
    assert call(a, dtype, 4096, 1 << 40, None) == status
    assert size(a, dtype) == 0


def test_attention_of_nothing_and_a_missing_problem():
    assert lib.sna_attention_forward(None, 1, None, 0, None) == 1 and lib.sna_attention_backward(None, 1, None, 0, None) == 1
    assert lib.sna_attention_forward(attention(B=0), 1, None, 0, None) == 0 and lib.sna_attention_backward(attention(B=0), 1, None, 0, None) == 0
    assert lib.sna_attention_backward(attention(lse=None), 1, 4096, 1 << 40, None) == 1
