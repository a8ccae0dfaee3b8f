"""8-bit storage, its products and the gated projection in 64 bits, each with a bound of what the kernels' roundings may add up to.

Bounds.  A rounding to a type is off by at most `half` of the value: 2^-24 in fp32, 2^-8 in bf16.  A sum of k products, in fp32 and in any
order, is off by at most (k + 2) 2^-23 times the sum of the magnitudes (a product and an addition a term; twice the half step, because the
matrix unit need not round every addition to the nearest).  An activation g s(g) is off by 1.2 times the error of g (no slope here is beyond
1.13), and by 16 half steps of |g| for s (an exponential or erfc, a division, the argument); a slope by the error of g (no second derivative
is beyond 0.8) and by 64 half steps (1 - s where s is near 1 is multiplied by g and z', up to 48)."""
from __future__ import annotations

import math

import torch

STEP = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def padded(cols):
    return -(-cols // 128) * 128


def stored(x):
    """(codes as whole numbers, scales) of fp32 or bf16 rows, by the definition: binary32 operations, each emulated from binary64."""
    x = x.double()
    codes, scales = torch.zeros_like(x), torch.zeros(x.shape[0], dtype=torch.float64, device=x.device)
    if x.numel() == 0:
        return codes, scales
    top = x.abs().amax(1)
    broken = ~torch.isfinite(x).all(1)
    some = (top >= 2.0 ** -100) & ~broken
    factor = (127.0 / top[some]).float().double()
    codes[some] = torch.round((x[some] * factor[:, None]).float().double())
    scales[some] = (top[some] / 127.0).float().double()
    scales[broken] = math.nan
    return codes, scales


def taken_apart(m):
    """(codes, their padding, scales) of a Q8Matrix as they lie."""
    width = padded(m.cols)
    codes = m.data[:m.rows * width].view(torch.int8).view(m.rows, width)
    return codes[:, :m.cols].double(), codes[:, m.cols:], m.data[m.rows * width:].view(torch.float32).double()


def mm(a, b):
    return torch.mm(a.contiguous(), b.contiguous())


def q8_product(a, b, bias):
    """(a b^T + bias, bound before the result's rounding) of (codes, scales) pairs."""
    sums = mm(a[0], b[0].t()) * (a[1][:, None] * b[1][None, :])
    bias = torch.zeros(b[0].shape[0], dtype=torch.float64, device=sums.device) if bias is None else bias.double()
    y = sums + bias
    # the integer sum, the scales' product and theirs with the sum are rounded, and the addition
    return y, 5 * STEP * (sums.abs() + bias.abs())


def dense_product(x, w, bias):
    x, w = x.double(), w.double()
    y, bound = mm(x, w.t()), (x.shape[1] + 2) * 2 * STEP * mm(x.abs(), w.abs().t())
    if bias is not None:
        y = y + bias.double()
        bound = bound + STEP * (y.abs() + bias.double().abs())
    return y, bound


def activation(g, act):
    """(act(g), act'(g)) in 64 bits."""
    if act == "silu":
        s = torch.special.expit(g)
        return g * s, s + g * s * torch.special.expit(-g)
    if act == "gelu":
        s = 0.5 * torch.special.erfc(-g / math.sqrt(2.0))
        return g * s, s + g * torch.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)
    z, turn = math.sqrt(8.0 / math.pi) * (g + 0.044715 * g ** 3), math.sqrt(8.0 / math.pi) * (1 + 3 * 0.044715 * g * g)
    s = torch.special.expit(z)
    return g * s, s + g * turn * s * torch.special.expit(-z)


def gated(gate, up, act, dtype):
    """(h, bound) of (value, bound) pairs, rounded to dtype."""
    (g, eg), (u, eu) = gate, up
    a = activation(g, act)[0]
    ea = 1.2 * eg + 16 * STEP * (g.abs() + eg)
    h = a * u
    bound = ea * (u.abs() + eu) + a.abs() * eu
    return h, bound + (HALF[dtype] + 2 * STEP) * (h.abs() + bound)


def gated_backward(dh, x, wg, wu, bg, bu, act, rests=False):
    """Five (gradient, bound) pairs; `rests`: the gradients of gate and up are two values of x's type each between the products, twice as many to add."""
    dtype, half = x.dtype, HALF[x.dtype]
    held, times = (half * half, 2 * (1 + 2 * half)) if rests else (half, 1)      # rests are up to `half` of the values: so much more to add
    g, eg = dense_product(x, wg, bg)
    u, eu = dense_product(x, wu, bu)
    a, slope = activation(g, act)
    dh, x, wg, wu = dh.double(), x.double(), wg.double(), wu.double()
    dg, du = dh * u * slope, dh * a
    e_slope = eg + 64 * STEP * (1 + eg)
    edg = dh.abs() * ((u.abs() + eu) * e_slope + slope.abs() * eu) + 4 * STEP * dg.abs()
    edu = dh.abs() * (1.2 * eg + 16 * STEP * (g.abs() + eg)) + 2 * STEP * du.abs()
    t, n = x.shape[0], wg.shape[0]

    def rounded(y, bound, to=half):
        return y, bound + to * (y.abs() + bound)

    _, edg_r = rounded(dg, edg, held)                            # as the products take them
    _, edu_r = rounded(du, edu, held)
    dx = mm(dg, wg) + mm(du, wu)
    ex = mm(edg_r, wg.abs()) + mm(edu_r, wu.abs()) + (2 * n * times + 2) * 2 * STEP * (mm(dg.abs() + edg_r, wg.abs()) + mm(du.abs() + edu_r, wu.abs()))

    def weight(d, ed):
        return rounded(mm(d.t(), x), mm(ed.t(), x.abs()) + (t * times + 2) * 2 * STEP * mm((d.abs() + ed).t(), x.abs()))

    def bias(d, ed):
        return rounded(d.sum(0), ed.sum(0) + (t + 2) * STEP * (d.abs() + ed).sum(0))

    return [rounded(dx, ex), weight(dg, edg_r), weight(du, edu_r), bias(dg, edg), bias(du, edu)]


def check(got, want, bound, what=""):
    got = got.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    broken = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got) | torch.isinf(got), broken), f"{what}: {int((~torch.isfinite(got)).sum())} values are no numbers, {int(broken.sum())} should be"
    off = torch.where(broken, torch.zeros_like(want), (got - want).abs() - bound)
    if off.numel():
        assert float(off.max()) <= 0, f"{what}: off by {float((got - want).abs().nan_to_num().max())}, {int((off > 0).sum())} of {off.numel()} beyond their bounds"
