"""Plain 64-bit forms of the microscaled formats and their products, for the tests alone (CPU, numpy and torch)."""
import math

import numpy as np
import torch

MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# the smallest normal numbers' half step: what a rounding into the subnormals may be off by
HALF_LEAST = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def mx4_blocks(cols):
    return (cols + 255) // 256 * 8


def ckpt8_blocks(cols):
    return (cols + 31) // 32


def _in_blocks(x, blocks):
    """float64 [rows][blocks][32], zeros beyond the columns, and the exponents of the largest finite magnitudes (-9999: none)."""
    rows, cols = x.shape
    b = np.zeros((rows, blocks * 32))
    b[:, :cols] = x
    b = b.reshape(rows, blocks, 32)
    finite = np.where(np.isfinite(b), np.abs(b), 0.0)
    peak = finite.max(2)
    _, e = np.frexp(peak)
    return b, np.where(peak > 0, e - 1, -9999)


def mx4_quantize(x, mode="even", draws=None):
    """x [rows][cols] -> (codes uint8 [rows][16 B], scales uint8 [rows][B], zeros, clipped)."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    blocks = mx4_blocks(cols)
    b, e = _in_blocks(x, blocks)
    byte = np.clip(e + 125, 2, 252)
    b = np.where(np.isnan(b), 0.0, b)
    t = np.abs(b) / np.exp2(byte - 127.0)[:, :, None]
    grid = np.append(MAGNITUDES, 8.0)                     # 8 does not exist: it saturates
    low = np.clip(np.searchsorted(grid, t, side="right") - 1, 0, 7)
    gap = grid[low + 1] - grid[low]
    part = (np.minimum(t, 8.0) - grid[low]) / gap
    if mode == "even":
        up = (part > 0.5) | ((part == 0.5) & (low % 2 == 1))
    elif mode == "away":
        up = part >= 0.5
    else:
        d = np.zeros((rows, blocks * 32))
        d[:, :cols] = draws.reshape(rows, cols)
        up = d.reshape(b.shape) / 2.0 ** 32 < part
    code = low + up
    real = (np.arange(blocks * 32) < cols).reshape(1, blocks, 32)
    zeros, clipped = int(((code == 0) & real).sum()), int(((code > 7) & real).sum())
    code = np.minimum(code, 7) | np.where(b < 0, 8, 0)
    code = code.reshape(rows, -1).astype(np.uint8)
    return code[:, 0::2] | (code[:, 1::2] << 4), byte.astype(np.uint8), zeros, clipped


def mx4_values(codes, scales, cols):
    codes, scales = np.asarray(codes), np.asarray(scales, np.float64)
    rows = scales.shape[0]
    code = np.stack([codes & 15, codes >> 4], 2).reshape(rows, -1)
    v = MAGNITUDES[code & 7] * np.where(code & 8, -1.0, 1.0)
    return (v * np.repeat(np.exp2(scales - 127), 32, 1))[:, :cols]


def ckpt8_quantize(x, mode="even", draws=None):
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    blocks = ckpt8_blocks(cols)
    b, e = _in_blocks(x, blocks)
    byte = np.clip(e + 127, 7, 254)
    t = np.where(np.isnan(b), 0.0, b) / np.exp2(byte - 133.0)[:, :, None]
    t = np.clip(t, -1000, 1000)
    if mode == "even":
        q = np.rint(t)
    elif mode == "away":
        q = np.copysign(np.floor(np.abs(t) + 0.5), t)
    else:
        d = np.zeros((rows, blocks * 32))
        d[:, :cols] = draws.reshape(rows, cols)
        q = np.floor(t) + (d.reshape(b.shape) / 2.0 ** 32 < t - np.floor(t))
    return np.clip(q, -127, 127).reshape(rows, -1).astype(np.int8), byte.astype(np.uint8)


def ckpt8_values(codes, scales, cols):
    v = np.asarray(codes, np.float64) * np.repeat(np.exp2(np.asarray(scales, np.float64) - 133), 32, 1)
    return v[:, :cols]


def act(h, name):
    """Activation function in 64 bits and the argument of its logistic factor (its rounding error grows with it)."""
    h = np.asarray(h, np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        if name == "relu":
            return np.where(h < 0, 0.0, h), np.zeros_like(h)
        if name == "none":
            return h, np.zeros_like(h)
        z = h if name == "silu" else 2 * math.sqrt(2 / math.pi) * (h + 0.044715 * h ** 3)
        return h / (1 + np.exp(-z)), np.abs(z)


def act_slope(h, name):
    h = np.asarray(h, np.float64)
    if name == "relu":
        return (h > 0).astype(np.float64)
    if name == "none":
        return np.ones_like(h)
    with np.errstate(over="ignore", invalid="ignore"):
        c = 2 * math.sqrt(2 / math.pi)
        z = h if name == "silu" else c * (h + 0.044715 * h ** 3)
        dz = np.ones_like(h) if name == "silu" else c * (1 + 3 * 0.044715 * h * h)
        s = 1 / (1 + np.exp(-z))
        return np.where(np.abs(z) > 700, (h > 0).astype(np.float64), s + h * s * (1 - s) * dz)


def act_error(y, z):
    """How far an activation function's result y, computed in 32 bits, may be off before its rounding.  z, the argument of the
    logistic factor, is off by a few half steps of its own size (at most 8: the polynomial's four operations, the
    constants, the product with log2 e); exp turns that into the relative error 8 |z| 2^-24; sum, reciprocal and product
    add less than 8 half steps.  (Where exp overflows, beyond 88, the result is below 1e-36 in magnitude.)"""
    return np.where(z > 87, 1e-35 + np.abs(y) * 2.0 ** -20, np.abs(y) * (8 * z + 8) * 2.0 ** -24) if np.ndim(z) else z


def product_error(sizes, count):
    """How far a sum of `count` products in 32 bits may be off in any order, rounded or cut: `sizes` is the sum of the
    products' magnitudes, each addition is off by at most a step (2^-23) of its result."""
    return (count + 2) * 2.0 ** -23 * sizes


def close(got, want, error, dtype):
    """got (a torch tensor of dtype) is want, off by at most `error` before its last rounding to dtype."""
    got = got.detach().cpu().double().numpy()
    bound = error + (np.abs(want) + error) * HALF_STEP[dtype] + HALF_LEAST[dtype]
    top = float(torch.finfo(dtype).max)
    fine = (np.abs(got - want) <= bound) | (np.isnan(got) & np.isnan(want)) | ((np.abs(want) + bound >= top) & (np.abs(got) >= top * (1 - 2.0 ** -7)) & (np.sign(got) == np.sign(want)))
    bad = np.argwhere(~fine)
    assert not len(bad), "%d of %d are off, first at %s: got %r, want %r, bound %r" % (
        len(bad), fine.size, bad[0], got[tuple(bad[0])], want[tuple(bad[0])], np.broadcast_to(bound, want.shape)[tuple(bad[0])])
