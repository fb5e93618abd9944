"""Plain numpy / float64 forms of the 8-bit layer and of the norms around it, for the tests."""

import numpy as np
import torch

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
CODES = {"fp16": 0, "fp32": 1, "bf16": 2}


def quantize_rows(x):
    """(q int8, scale fp32) of x [T x n] (float32 numpy), to the bit: the product with the fp32 factor is exact in 64 bits."""
    x = np.asarray(x, np.float32)
    top = np.abs(x).max(1)                                   # (NaN where a row has one)
    bad = ~(top < np.inf)
    none = top < np.float32(2.0 ** -100)
    with np.errstate(all="ignore"):
        factor = np.where(bad | none, np.float32(0), (np.float32(1) / top) * np.float32(127)).astype(np.float32)
        scale = np.where(bad, np.float32(np.nan), np.where(none, np.float32(0), top * (np.float32(1) / np.float32(127)))).astype(np.float32)
        q = np.rint(x.astype(np.float64) * factor.astype(np.float64)[:, None])
    q[bad | none] = 0
    return q.astype(np.int8), scale


def random_triple(rng, out, inn, V, M):
    """An int8 V:N:M weight: (values, meta, colidx, scale, dense int64 [out x in]); every value of int8 occurs, -128 too.  The
    values at pad columns are not zero: they count as zero whatever they are."""
    R, B = -(-out // V), -(-inn // M)
    col = np.sort(rng.random((R, B, M)).argsort(2)[:, :, :4], 2).astype(np.uint8)
    pairs = np.array([(0, 1), (0, 2), (0, 3), (1, 2), (1, 3), (2, 3)])
    pos = pairs[rng.integers(0, 6, (R * V, B))]
    values = rng.integers(-128, 128, (R * V, B, 2)).astype(np.int8)
    values[out:] = 0
    nibble = (pos[..., 0] | pos[..., 1] << 2).astype(np.uint8)
    if B % 2:
        nibble = np.concatenate([nibble, np.full((R * V, 1), 4, np.uint8)], 1)
    meta = (nibble[:, 0::2] | nibble[:, 1::2] << 4).astype(np.uint8)
    kept = np.take_along_axis(np.repeat(col, V, 0).astype(np.int64), pos, 2) + np.arange(B)[None, :, None] * M
    dense = np.zeros((R * V, B * M), np.int64)
    np.put_along_axis(dense, kept.reshape(R * V, -1), values.reshape(R * V, -1).astype(np.int64), 1)
    scale = rng.uniform(1e-4, 1e-2, out).astype(np.float32)
    return values, meta, col, scale, dense[:out, :inn]


def product(q, scale_x, dense, scale_w, bias, dtype):
    """The product's result to the bit, as a torch tensor of `dtype`: exact sums, then fp32 operations rounded one by one."""
    sums = q.astype(np.float64) @ dense.T.astype(np.float64)           # below 2^53: exact
    with np.errstate(all="ignore"):
        y = (sums.astype(np.float32) * scale_w[None, :]) * scale_x[:, None]
        if bias is not None:
            y = y + bias.astype(np.float32)[None, :]
    return torch.from_numpy(y).to(TYPES[dtype])


def normed(v, kind, w, b, eps):
    """(result, mean, r, magnitude of what was added up on the way) of a norm over the rows of v, in float64 (torch)."""
    if kind == "none":
        return v, torch.zeros_like(v[:, :1]), torch.ones_like(v[:, :1])
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    r = 1.0 / torch.sqrt((v - mean).square().mean(1, keepdim=True) + eps)
    x = (v - mean) * r
    x = x * w if w is not None else x
    return (x + b if b is not None else x), mean, r


def norm_magnitude(v, mag, kind, w, b, eps):
    """A bound of the size of the terms behind each normalised value: errors of fp32 arithmetic are a small number of its
    roundings.  `mag`: the same for v."""
    if kind == "none":
        return mag
    x, mean, r = normed(v, kind, None, None, eps)
    spread = (mag + (mag.mean(1, keepdim=True) if kind == "layer" else 0.0) + x.abs() * mag.square().mean(1, keepdim=True).sqrt()) * r
    spread = spread * w.abs() if w is not None else spread
    return spread + b.abs() if b is not None else spread


def residual_norm(h, y, gate_rows, scale, post, pre):
    """(h', x, stats, magnitude of h', magnitude of x) in float64; post, pre = (kind, weight, bias, eps)."""
    p, ym, yr = normed(y, *post) if y is not None else (None, torch.zeros_like(h[:, :1]), torch.ones_like(h[:, :1]))
    new, mag = scale * h, (scale * h).abs()
    if y is not None:
        g = 1.0 if gate_rows is None else gate_rows
        new = new + g * p
        pm = norm_magnitude(y, y.abs(), *post)
        mag = mag + (pm if gate_rows is None else gate_rows.abs() * pm)
    x, hm, hr = normed(new, *pre)
    return new, x, torch.cat([ym, yr, hm, hr], 1), mag, norm_magnitude(new, mag, *pre)
