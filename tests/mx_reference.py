"""Microscaled storage, its product and layer norm in binary64, by numpy: what the kernels' tests compare with, and the
bounds within which a binary32 computation has to stay."""
from __future__ import annotations

import numpy as np

from np_quantiser import philox4x32_10_np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
U32 = 2.0 ** -24                                   # half a step of binary32, relative
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def philox_halves(rows, cols, seed, tensor_id):
    """The 16 random bits of every value, [rows][cols]: Philox4x32-10, a block for eight rows of a column."""
    at = np.arange(-(-rows // 8) * cols, dtype=np.uint64)
    c = philox4x32_10_np(at & np.uint64(0xFFFFFFFF), at >> np.uint64(32), tensor_id & 0xFFFFFFFF, tensor_id >> 32,
                         seed & 0xFFFFFFFF, seed >> 32)
    c = [np.broadcast_to(w, at.shape) for w in c]
    out = np.empty((-(-rows // 8) * 8, cols), dtype=np.int64)
    for i in range(8):
        out[i::8] = ((c[i // 2] >> np.uint64(16 * (i % 2))) & np.uint64(0xFFFF)).astype(np.int64).reshape(-1, cols)
    return out[:rows]


def padded(cols):
    return -(-cols // 256) * 256


def codes_and_scales(x, halves=None):
    """(codes [rows][padded cols], scale bytes [rows][padded cols / 32]) of a matrix of float32 values."""
    x = np.asarray(x, dtype=np.float32)
    rows, cols = x.shape
    width = padded(cols)
    v = np.zeros((rows, width), dtype=np.float64)
    v[:, :cols] = x
    negative = np.zeros((rows, width), dtype=bool)
    negative[:, :cols] = np.signbit(x)
    h = np.zeros((rows, width), dtype=np.int64)
    if halves is not None:
        h[:, :cols] = halves
    blocks = np.abs(v).reshape(rows, -1, 32)
    broken = ~np.isfinite(blocks).all(2)
    blocks = np.where(broken[..., None], 0.0, blocks)
    top = blocks.max(2)
    exponent = np.where(top > 0, np.frexp(top)[1] - 1, -10000)
    s = np.maximum(exponent - 2 + 127, 1)
    t = np.minimum(blocks * np.exp2(127.0 - s)[..., None], 6.0).reshape(rows, width)
    low = np.searchsorted(GRID, t, side="right") - 1
    low = np.minimum(low, 6)
    a, b = GRID[low], GRID[low + 1]
    if halves is None:
        up = (t - a > b - t) | ((t - a == b - t) & (low % 2 == 1))
    else:
        up = np.rint((t - a) / (b - a) * 2.0 ** 22) > 64 * h
    code = np.where(t >= 6.0, 7, low + up) | np.where(negative, 8, 0)
    dead = np.repeat(broken, 32, axis=1)
    return np.where(dead, 0, code).astype(np.uint8), np.where(broken, 255, s).astype(np.uint8)


def scale_positions(rows, width):
    r, b = np.arange(rows)[:, None], np.arange(width // 32)[None]
    return (r // 32 * (width // 256) + b // 8) * 256 + b % 8 // 4 * 128 + r % 32 * 4 + b % 4


def stored(x, halves=None):
    """(the stored form's bytes, which of them are specified)"""
    codes, scales = codes_and_scales(x, halves)
    rows, width = codes.shape
    data = np.zeros(rows * width // 2 + -(-rows // 32) * 32 * (width // 32), dtype=np.uint8)
    known = np.zeros(data.size, dtype=bool)
    data[:rows * width // 2] = (codes[:, 0::2] | codes[:, 1::2] << 4).reshape(-1)
    known[:rows * width // 2] = True
    at = rows * width // 2 + scale_positions(rows, width)
    data[at], known[at] = scales, True
    return data, known


def restored(data, rows, cols):
    """The values that a stored matrix stands for, in binary64."""
    data, width = np.asarray(data), padded(cols)
    packed = data[:rows * width // 2].reshape(rows, width // 2)
    code = np.empty((rows, width), dtype=np.uint8)
    code[:, 0::2], code[:, 1::2] = packed & 15, packed >> 4
    s = data[rows * width // 2:][scale_positions(rows, width)].astype(np.int64)
    scale = np.where(s == 255, np.nan, np.exp2(s - 127.0))
    v = GRID[code & 7] * np.where(code & 8, -1.0, 1.0)
    return (v * np.repeat(scale, 32, axis=1))[:, :cols]


def product(a, b, bias=None):
    """(a b^T + bias, the bound of a binary32 computation of it without the last rounding): products of 4-bit values are
    exact, a sum of 32 terms and more is rounded once per matrix instruction and once per joined part."""
    y, size = a @ b.T, np.abs(a) @ np.abs(b).T
    if bias is not None:
        y, size = y + bias, size + np.abs(bias)
    return y, (a.shape[1] / 32 + 32) * U32 * size


def layer_norm(x, weight, bias, eps):
    """(y, mean, rstd, bounds of the three without y's last rounding).  A sum of n terms in a tree of threads has a depth of
    64 additions for rows in registers, and n / 1024 more for longer ones."""
    n = x.shape[1]
    depth = 64 + n / 1024
    mean = x.mean(1, keepdims=True)
    d = x - mean
    var = (d * d).mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(var + eps)
    d_mean = (depth + 1) * U32 * np.abs(x).mean(1, keepdims=True)
    d_value = d_mean + U32 * np.abs(d)
    d_var = (2 * np.abs(d) * d_value + d_value ** 2).mean(1, keepdims=True) + (depth + 2) * U32 * var
    d_rstd = rstd * (0.5 * d_var / (var + eps) * 1.01 + 4 * U32)
    h = d * rstd
    y = h * weight + bias
    d_y = np.abs(weight) * (d_value * rstd + np.abs(d) * d_rstd + U32 * np.abs(h)) * 1.01 + 2 * U32 * (np.abs(y) + np.abs(bias))
    return y, mean[:, 0], rstd[:, 0], d_y, d_mean[:, 0], d_rstd[:, 0]


def layer_norm_backward(dy, x, mean, rstd, weight):
    """(dx, dweight, dbias, their bounds without the last rounding); the statistics are inputs.  The columns' sums have a depth of
    rows / 256 additions in a workgroup and 256 more where those are joined."""
    rows, n = x.shape
    depth, depth_rows = 64 + n / 1024, rows / 256 + 300
    h = (x - mean[:, None]) * rstd[:, None]
    g = dy * weight
    s1, s2 = g.mean(1, keepdims=True), (g * h).mean(1, keepdims=True)
    dx = rstd[:, None] * (g - s1 - h * s2)
    d_s1 = (depth + 3) * U32 * np.abs(g).mean(1, keepdims=True)
    d_s2 = (depth + 6) * U32 * np.abs(g * h).mean(1, keepdims=True)
    d_dx = np.abs(rstd[:, None]) * (d_s1 + np.abs(h) * d_s2 + 6 * U32 * (np.abs(g) + np.abs(s1) + np.abs(h * s2))) * 1.01
    return (dx, (dy * h).sum(0), dy.sum(0), d_dx, (depth_rows + 3) * U32 * np.abs(dy * h).sum(0), depth_rows * U32 * np.abs(dy).sum(0))
