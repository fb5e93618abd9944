"""int8 products of more tokens and of more rows than one launch has room for, bit for bit (computed on the device in fp64)."""

import pytest
import torch

import paper_2410_16135_amd as vnm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def layer(out, inn, V, seed):
    """An int8 layer at M = 4 (every column of a block is kept) and its weight, dense in int8."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    R, B = -(-out // V), inn // 4
    assert inn % 8 == 0
    pairs = torch.tensor([(0, 1), (0, 2), (0, 3), (1, 2), (1, 3), (2, 3)], device=DEV)
    pos = pairs[torch.randint(0, 6, (R * V, B), generator=g, device=DEV)]
    values = torch.randint(-128, 128, (R * V, B, 2), generator=g, device=DEV, dtype=torch.int8)
    values[out:] = 0
    nibble = (pos[..., 0] | pos[..., 1] << 2).to(torch.uint8)
    dense = torch.zeros(R * V, B, 4, dtype=torch.int8, device=DEV).scatter_(2, pos, values).view(R * V, inn)[:out]
    scale = torch.rand(out, generator=g, device=DEV) * 1e-2 + 1e-4
    col = torch.arange(4, dtype=torch.uint8, device=DEV).repeat(R * B)
    c = vnm.CompressedI8(values.view(-1), (nibble[:, 0::2] | nibble[:, 1::2] << 4).reshape(-1), col, None, scale, out, inn, V, 4)
    return vnm.vnm_pack_i8(c), dense


def activations(T, inn, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    q = torch.randint(-128, 128, (T, inn), generator=g, device=DEV, dtype=torch.int8)
    return q, torch.rand(T, generator=g, device=DEV) * 1e-1 + 1e-3


def same(y, q, sx, dense, sw, bias):
    """Whether y holds the product's bits: exact sums, then single fp32 operations."""
    want = ((q.double() @ dense.double().t().contiguous()).float() * sw[None]) * sx[:, None]
    return torch.equal(y, (want + bias.float()[None] if bias is not None else want).to(y.dtype))


def test_more_tiles_of_tokens_than_a_grid_has_rows():
    T, out, inn = 65535 * 128 + 300, 8, 16
    c, dense = layer(out, inn, 64, 1)
    q, sx = activations(T, inn, 2)
    bias = torch.randn(out, device=DEV).half()
    assert vnm.vnm_spmm_i8_workspace_bytes(T, c) > 0                  # the many-token kernels
    y = vnm.vnm_spmm_i8(q, sx, c, bias=bias)
    for t in range(0, T, 1 << 20):
        s = slice(t, t + (1 << 20))
        assert same(y[s], q[s], sx[s], dense, c.scale, bias), t


def test_more_row_blocks_than_a_grid_has_rows():
    T, out, inn = 3, 65535 * 8 * 64 + 70, 8
    c, dense = layer(out, inn, 128, 3)
    q, sx = activations(T, inn, 4)
    rows = torch.zeros(T, 16, dtype=torch.int8, device=DEV)           # rows 16 bytes aligned
    rows[:, :inn] = q
    bias = torch.randn(out, device=DEV).half()
    y = vnm.vnm_spmm_i8_staged(vnm.vnm_stage_q(rows[:, :inn], 4), sx, c, bias=bias, out_dtype=torch.float32)
    for o in range(0, out, 1 << 22):
        s = slice(o, o + (1 << 22))
        assert same(y[:, s], q, sx, dense[s], c.scale[s], bias[s]), o
