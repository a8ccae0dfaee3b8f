"""Microscaled storage and layer norm without a GPU: sizes, the layout's definition, refusals before any launch."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

import mx_reference as R
from paper_2510_11400_amd import api

FAKE = 0x10000  # an aligned non-NULL address; never dereferenced because validation fails first
BIG = 1 << 40
LIB = api.raw_library()


@pytest.mark.parametrize("rows, cols", [(0, 5), (5, 0), (1, 1), (1, 256), (31, 257), (32, 256), (33, 255), (8192, 768), (2 ** 31 - 256, 1)])
def test_sizes(rows, cols):
    width = -(-cols // 256) * 256
    assert api.mx_scales_offset(rows, cols) == rows * width // 2
    assert api.mx_bytes(rows, cols) == rows * width // 2 + -(-rows // 32) * 32 * width // 32


def test_sizes_of_bad_shapes_are_zero():
    for rows, cols in ((-1, 4), (4, -1), (2 ** 31 - 255, 1), (1, 2 ** 31)):
        assert api.mx_bytes(rows, cols) == 0 and api.mx_scales_offset(rows, cols) == 0
        assert LIB.fh_layer_norm_backward_workspace_bytes(rows, cols) == 0
    assert LIB.fh_layer_norm_backward_workspace_bytes(4, 0) == 0
    assert LIB.fh_mx_matmul_workspace_bytes(4, 4, -1) == 0 and LIB.fh_mx_matmul_workspace_bytes(-4, 4, 1) == 0


def test_scale_positions_are_a_permutation():
    at = R.scale_positions(64, 768)
    assert sorted(at.reshape(-1)) == list(range(64 * 24))


def test_the_reference_rounds_as_the_definition_says():
    """Every code's value restores to itself, midpoints go to the even code, blocks of zeros and broken blocks as defined."""
    x = np.zeros((4, 32), dtype=np.float32)
    x[0, :8], x[0, 8:16] = R.GRID * 4, -R.GRID * 4
    x[1, :9] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.9, 4.0]
    x[3, 5] = np.inf
    codes, scales = R.codes_and_scales(x)
    assert list(codes[0, :16]) == list(range(8)) + list(range(8, 16)) and scales[0, 0] == 129
    assert list(codes[1, :9]) == [0, 2, 2, 4, 4, 6, 6, 7, 6] and scales[1, 0] == 127
    assert scales[2, 0] == 1 and not codes[2].any()
    assert scales[3, 0] == 255 and not codes[3].any() and scales[3, 1] == 1
    data, _ = R.stored(x)
    back = R.restored(data, 4, 32)
    assert np.array_equal(back[0], x[0]) and np.isnan(back[3]).all() and not back[2].any()


def test_the_reference_rounds_up_as_often_as_the_fraction_says():
    rows, cols = 4096, 8
    x = np.full((rows, cols), 0.8, dtype=np.float32)
    x[:, 0] = 4.0
    halves = R.philox_halves(rows, cols, 7, 3)
    back = R.restored(R.stored(x, halves)[0], rows, cols)
    assert set(np.unique(back[:, 1:])) == {0.5, 1.0}
    # 28672 draws of up with probability 0.6: six standard deviations are 0.017
    assert abs((back[:, 1:] == 1.0).mean() - 0.6) < 0.018


def _quantize(x=FAKE, dtype=0, rows=4, cols=40, stride=40, rounding=0, a=FAKE, a_cap=BIG, b=FAKE, b_cap=BIG):
    return LIB.fh_mx_quantize(x, dtype, rows, cols, stride, rounding, 0, 0, a, a_cap, b, b_cap, None)


def test_quantize_refusals():
    assert _quantize(dtype=2) == 2 and _quantize(dtype=-1) == 2
    assert _quantize(rounding=2) == 5
    for bad in (dict(rows=-1), dict(cols=-1, stride=0), dict(stride=39), dict(rows=2 ** 31), dict(stride=2 ** 31 + 1)):
        assert _quantize(**bad) == 11, bad
    assert _quantize(x=None) == 1 and _quantize(a=None, b=None) == 1
    assert _quantize(x=FAKE + 2) == 8 and _quantize(x=FAKE + 1, dtype=1) == 8 and _quantize(a=FAKE + 8) == 8 and _quantize(b=FAKE + 4) == 8
    assert _quantize(a_cap=api.mx_bytes(4, 40) - 1) == 7 and _quantize(b_cap=api.mx_bytes(40, 4) - 1) == 7
    assert _quantize(rows=0, x=None, a=None, b=None) == 0 and _quantize(cols=0, stride=0, x=None, a=None, b=None) == 0


def _dequantize(m=FAKE, cap=BIG, rows=4, cols=40, dtype=0, out=FAKE, stride=40, out_cap=BIG):
    return LIB.fh_mx_dequantize(m, cap, rows, cols, dtype, out, stride, out_cap, None)


def test_dequantize_refusals():
    assert _dequantize(dtype=9) == 2
    assert _dequantize(rows=-1) == 11 and _dequantize(stride=39) == 11
    assert _dequantize(m=None) == 1 and _dequantize(out=None) == 1
    assert _dequantize(m=FAKE + 8) == 8 and _dequantize(out=FAKE + 2) == 8
    assert _dequantize(cap=api.mx_bytes(4, 40) - 1) == 7
    assert _dequantize(stride=50, out_cap=(3 * 50 + 40) * 4 - 1) == 7
    assert _dequantize(rows=0, m=None, out=None) == 0


def _matmul(**change):
    p = api.fh_mx_product(FAKE, BIG, FAKE, BIG, 5, 7, 40, None, 0, 0, FAKE, 7, BIG, FAKE, BIG, 0)
    for name, v in change.items():
        setattr(p, name, v)
    return LIB.fh_mx_matmul(ctypes.byref(p), None)


def test_matmul_refusals():
    assert LIB.fh_mx_matmul(None, None) == 1
    assert _matmul(out_dtype=2) == 2 and _matmul(bias_dtype=5) == 2
    for bad in (dict(m=-1), dict(n=-1), dict(k=-1), dict(stride=6), dict(k=2 ** 24 + 1), dict(m=2 ** 31), dict(stride=2 ** 31 + 1)):
        assert _matmul(**bad) == 11, bad
    assert _matmul(reserved=1) == 12
    assert _matmul(a=None) == 1 and _matmul(b=None) == 1 and _matmul(out=None) == 1
    assert _matmul(a=FAKE + 8) == 8 and _matmul(b=FAKE + 1) == 8 and _matmul(out=FAKE + 2) == 8 and _matmul(bias=FAKE + 2) == 8
    assert _matmul(a_cap=api.mx_bytes(5, 40) - 1) == 7 and _matmul(b_cap=api.mx_bytes(7, 40) - 1) == 7
    assert _matmul(out_cap=5 * 7 * 4 - 1) == 7 and _matmul(stride=9, out_cap=(4 * 9 + 7) * 4 - 1) == 7
    assert _matmul(m=0, a=None, out=None) == 0 and _matmul(n=0, stride=0, b=None, out=None) == 0


def test_matmul_workspace_is_asked_for():
    """A product that needs one is refused without, or with too little."""
    m, n, k = 96, 96, 1 << 20
    need = LIB.fh_mx_matmul_workspace_bytes(m, n, k)
    if not need:
        pytest.skip("no product of these sizes is split")
    assert _matmul(m=m, n=n, k=k, stride=n, workspace=None) == 1
    assert _matmul(m=m, n=n, k=k, stride=n, workspace_cap=need - 1) == 7
    assert _matmul(m=m, n=n, k=k, stride=n, workspace=FAKE + 4) == 8


def _norm(x=FAKE, dtype=0, rows=4, cols=40, xs=40, w=FAKE, b=FAKE, p=0, eps=1e-5, y=FAKE, ys=40, cap=BIG, mean=FAKE, rstd=FAKE):
    return LIB.fh_layer_norm(x, dtype, rows, cols, xs, w, b, p, eps, y, ys, cap, mean, rstd, None)


def test_layer_norm_refusals():
    assert _norm(dtype=2) == 2 and _norm(p=2) == 2
    for bad in (dict(rows=-1), dict(cols=0, xs=0, ys=0), dict(xs=39), dict(ys=39), dict(xs=2 ** 31 + 1)):
        assert _norm(**bad) == 11, bad
    assert _norm(eps=-1e-9) == 12 and _norm(eps=float("nan")) == 12
    assert _norm(x=None) == 1 and _norm(y=None) == 1
    for bad in (dict(x=FAKE + 2), dict(y=FAKE + 2), dict(w=FAKE + 2), dict(b=FAKE + 1), dict(mean=FAKE + 2), dict(rstd=FAKE + 2)):
        assert _norm(**bad) == 8, bad
    assert _norm(cap=4 * 40 * 4 - 1) == 7
    assert _norm(rows=0, x=None, y=None) == 0


def _norm_mx(x=FAKE, dtype=0, rows=4, cols=40, xs=40, w=FAKE, b=FAKE, p=0, eps=1e-5, rounding=0, a=FAKE, a_cap=BIG, c=FAKE, c_cap=BIG,
             mean=FAKE, rstd=FAKE):
    return LIB.fh_layer_norm_mx(x, dtype, rows, cols, xs, w, b, p, eps, rounding, 0, 0, a, a_cap, c, c_cap, mean, rstd, None)


def test_layer_norm_mx_refusals():
    assert _norm_mx(dtype=2) == 2 and _norm_mx(p=3) == 2 and _norm_mx(rounding=7) == 5
    for bad in (dict(rows=-1), dict(cols=0, xs=0), dict(xs=39)):
        assert _norm_mx(**bad) == 11, bad
    assert _norm_mx(eps=-1.0) == 12
    assert _norm_mx(x=None) == 1 and _norm_mx(a=None, c=None) == 1
    assert _norm_mx(mean=None) == 1 and _norm_mx(rstd=None) == 1 and _norm_mx(c=None, rounding=1, mean=None) == 1
    assert _norm_mx(a=FAKE + 8) == 8 and _norm_mx(c=FAKE + 8) == 8 and _norm_mx(w=FAKE + 2) == 8 and _norm_mx(mean=FAKE + 1) == 8
    assert _norm_mx(a_cap=api.mx_bytes(4, 40) - 1) == 7 and _norm_mx(c_cap=api.mx_bytes(40, 4) - 1) == 7
    assert _norm_mx(rows=0, x=None) == 0


def _backward(**change):
    p = api.fh_norm_backward(FAKE, FAKE, 40, 40, FAKE, FAKE, FAKE, 4, 40, 0, 0, FAKE, 40, BIG, FAKE, FAKE, FAKE, BIG)
    for name, v in change.items():
        setattr(p, name, v)
    return LIB.fh_layer_norm_backward(ctypes.byref(p), None)


def test_layer_norm_backward_refusals():
    assert LIB.fh_layer_norm_backward(None, None) == 1
    assert _backward(dtype=2) == 2 and _backward(p_dtype=2) == 2
    for bad in (dict(rows=-1), dict(cols=0), dict(dy_stride=39), dict(x_stride=39), dict(dx_stride=39), dict(cols=2 ** 31)):
        assert _backward(**bad) == 11, bad
    for name in ("dy", "x", "mean", "rstd", "workspace"):
        assert _backward(**{name: None}) == 1, name
    for name in ("dy", "x", "mean", "rstd", "weight", "dx", "dweight", "dbias", "workspace"):
        assert _backward(**{name: FAKE + 2}) == 8, name
    need = LIB.fh_layer_norm_backward_workspace_bytes(4, 40)
    assert need > 0 and _backward(workspace_cap=need - 1) == 7
    assert _backward(dx_cap=4 * 40 * 4 - 1) == 7
    assert _backward(rows=0, dweight=None, dbias=None, dy=None, x=None, dx=None, workspace=None) == 0


def test_the_binding_refuses_host_tensors_and_shapes():
    x = torch.zeros(4, 40)
    m = api.MxMatrix(torch.zeros(api.mx_bytes(4, 40), dtype=torch.uint8), 4, 40)
    for call in (lambda: api.fh_mx_quantize(x), lambda: api.fh_mx_dequantize(m), lambda: api.fh_mx_matmul(m, m),
                 lambda: api.fh_layer_norm(x), lambda: api.fh_layer_norm_mx(x),
                 lambda: api.fh_layer_norm_backward(x, x, x[:, 0], x[:, 0])):
        with pytest.raises(ValueError, match="device memory"):
            call()
    with pytest.raises(ValueError, match="forms"):
        api.fh_mx_quantize(x, "diagonal")


@pytest.mark.parametrize("rows, cols", [(0, 0), (0, 5), (5, 0), (1, 1), (33, 255), (8192, 768), (2 ** 31 - 256, 257), (3, 2 ** 31 - 256), (-1, 5), (5, -1),
                                        (2 ** 31 - 255, 1), (1, 2 ** 31)])
def test_the_binding_and_the_library_agree_on_sizes(rows, cols):
    assert api.mx_bytes(rows, cols) == LIB.fh_mx_bytes(rows, cols)
    assert api.mx_scales_offset(rows, cols) == LIB.fh_mx_scales_offset(rows, cols)


def _layer(backward=False, **change):
    a = api.fh_mx_layer(5, 40, 7, 0, 0, 1, 3, 0, 1e-5, 0, 0, FAKE, 40, FAKE, FAKE, FAKE, 40, FAKE, FAKE, FAKE, 7, FAKE, FAKE, FAKE, FAKE,
                        FAKE, BIG, FAKE, BIG, 0)
    for name, v in change.items():
        setattr(a, name, v)
    return (LIB.fh_mx_layer_backward if backward else LIB.fh_mx_layer_forward)(ctypes.byref(a), None)


@pytest.mark.parametrize("backward", [False, True])
def test_layer_refusals(backward):
    assert (LIB.fh_mx_layer_backward if backward else LIB.fh_mx_layer_forward)(None, None) == 1
    assert _layer(backward, dtype=2) == 2 and _layer(backward, p_dtype=-1) == 2 and _layer(backward, rounding=2) == 5
    for bad in (dict(tokens=-1), dict(features=0), dict(out_features=0), dict(tokens=2 ** 24 + 1), dict(features=2 ** 24 + 1), dict(x_stride=39),
                dict(weight_stride=39), dict(dy_stride=6), dict(x_stride=2 ** 31 + 1)):
        assert _layer(backward, **bad) == 11, bad
    for bad in (dict(norm=2), dict(needs=4), dict(needs=-1), dict(reserved=1), dict(eps=-1.0), dict(eps=float("nan"))):
        assert _layer(backward, **bad) == 12, bad
    needed = ("kept", "scratch", "dweight", "dy", "dx", "x") if backward else ("kept", "scratch", "x", "weight", "y")
    for name in needed:
        assert _layer(backward, **{name: None}) == 1, name
    aligned = ("x", "dy", "dx", "dweight", "norm_weight", "dnorm_weight", "dnorm_bias") if backward else ("x", "y", "weight", "bias", "norm_weight", "norm_bias")
    for name in aligned:
        assert _layer(backward, **{name: FAKE + 2}) == 8, name
    assert _layer(backward, kept=FAKE + 8) == 8 and _layer(backward, scratch=FAKE + 4) == 8
    assert _layer(backward, kept_cap=LIB.fh_mx_layer_kept_bytes(5, 40, 7) - 1) == 7 and _layer(backward, scratch_cap=100) == 7
    assert (_layer(True, needs=0, kept=None, scratch=None) if backward else _layer(tokens=0, x=None, y=None, kept=None)) == 0


def test_layer_sizes():
    assert LIB.fh_mx_layer_kept_bytes(0, 1, 1) >= 0
    for bad in ((-1, 4, 4), (4, 0, 4), (4, 4, 0), (2 ** 24 + 1, 4, 4)):
        assert LIB.fh_mx_layer_kept_bytes(*bad) == 0 and LIB.fh_mx_layer_scratch_bytes(*bad) == 0
    kept = LIB.fh_mx_layer_kept_bytes(100, 300, 70)
    assert kept >= 2 * 400 + api.mx_bytes(300, 100) + api.mx_bytes(300, 70)
    assert LIB.fh_mx_layer_scratch_bytes(100, 300, 70) >= max(api.mx_bytes(100, 300) + api.mx_bytes(70, 300), api.mx_bytes(100, 70) + api.mx_bytes(70, 100))


def test_layer_bias_gradient_refusals():
    assert _layer(True, dbias=FAKE + 2) == 8
    assert _layer(True, dbias=FAKE, needs=0, kept=None, scratch=None) == 1 and _layer(True, dbias=FAKE, needs=0, kept=None, dy=None) == 1
    assert _layer(True, dbias=FAKE, needs=0, kept=None, scratch_cap=LIB.fh_mx_layer_scratch_bytes(5, 40, 7) // 2) == 7
    # the partial sums of a long, wide gradient fit
    assert LIB.fh_mx_layer_scratch_bytes(2 ** 20, 1, 4096) >= api.mx_bytes(2 ** 20, 4096) + api.mx_bytes(4096, 2 ** 20) + 4096 * 4096 * 4
