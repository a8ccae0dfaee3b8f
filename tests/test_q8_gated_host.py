"""8-bit integer storage, its products and the gated projection without a GPU: sizes, refusals before any launch."""
from __future__ import annotations

import ctypes

import pytest
import torch

from paper_2510_11400_amd import api, layers

FAKE = 0x10000  # an aligned non-NULL address; never dereferenced because validation fails first
BIG = 1 << 40
LIB = api.raw_library()


@pytest.mark.parametrize("rows, cols", [(0, 0), (0, 5), (5, 0), (1, 1), (1, 128), (33, 129), (8192, 768), (2 ** 31 - 256, 257), (3, 2 ** 31 - 256)])
def test_sizes(rows, cols):
    width = -(-cols // 128) * 128
    assert api.q8_scales_offset(rows, cols) == LIB.fh_q8_scales_offset(rows, cols) == rows * width
    assert api.q8_bytes(rows, cols) == LIB.fh_q8_bytes(rows, cols) == (rows * width + 4 * rows if cols else 0)


@pytest.mark.parametrize("rows, cols", [(-1, 4), (4, -1), (2 ** 31 - 255, 1), (1, 2 ** 31 - 255)])
def test_sizes_of_bad_shapes_are_zero(rows, cols):
    assert api.q8_bytes(rows, cols) == LIB.fh_q8_bytes(rows, cols) == 0
    assert api.q8_scales_offset(rows, cols) == LIB.fh_q8_scales_offset(rows, cols) == 0


def _quantize(x=FAKE, dtype=0, rows=4, cols=40, stride=40, a=FAKE, cap=BIG):
    return LIB.fh_q8_quantize(x, dtype, rows, cols, stride, a, cap, None)


def test_quantize_refusals():
    assert _quantize(dtype=2) == 2 and _quantize(dtype=-1) == 2
    for bad in (dict(rows=-1), dict(cols=-1, stride=0), dict(stride=39), dict(rows=2 ** 31), dict(stride=2 ** 31 + 1)):
        assert _quantize(**bad) == 11, bad
    assert _quantize(x=None) == 1 and _quantize(a=None) == 1
    assert _quantize(x=FAKE + 2) == 8 and _quantize(x=FAKE + 1, dtype=1) == 8 and _quantize(a=FAKE + 8) == 8
    assert _quantize(cap=api.q8_bytes(4, 40) - 1) == 7
    assert _quantize(rows=0, x=None, a=None) == 0 and _quantize(cols=0, stride=0, x=None, a=None) == 0


def _dequantize(m=FAKE, cap=BIG, rows=4, cols=40, dtype=0, out=FAKE, stride=40, out_cap=BIG):
    return LIB.fh_q8_dequantize(m, cap, rows, cols, dtype, out, stride, out_cap, None)


def test_dequantize_refusals():
    assert _dequantize(dtype=9) == 2
    assert _dequantize(rows=-1) == 11 and _dequantize(stride=39) == 11
    assert _dequantize(m=None) == 1 and _dequantize(out=None) == 1
    assert _dequantize(m=FAKE + 8) == 8 and _dequantize(out=FAKE + 2) == 8
    assert _dequantize(cap=api.q8_bytes(4, 40) - 1) == 7
    assert _dequantize(stride=50, out_cap=(3 * 50 + 40) * 4 - 1) == 7
    assert _dequantize(rows=0, m=None, out=None) == 0


def _matmul(**change):
    p = api.fh_q8_product(FAKE, BIG, FAKE, BIG, 5, 7, 40, None, 0, 0, FAKE, 7, BIG, FAKE, BIG, 0)
    for name, v in change.items():
        setattr(p, name, v)
    return LIB.fh_q8_matmul(ctypes.byref(p), None)


def test_matmul_refusals():
    assert LIB.fh_q8_matmul(None, None) == 1
    assert _matmul(out_dtype=2) == 2 and _matmul(bias_dtype=5) == 2
    for bad in (dict(m=-1), dict(n=-1), dict(k=-1), dict(stride=6), dict(k=2 ** 17), dict(m=2 ** 31), dict(stride=2 ** 31 + 1)):
        assert _matmul(**bad) == 11, bad
    assert _matmul(reserved=1) == 12
    assert _matmul(a=None) == 1 and _matmul(b=None) == 1 and _matmul(out=None) == 1
    for bad in (dict(a=FAKE + 8), dict(b=FAKE + 1), dict(out=FAKE + 2), dict(bias=FAKE + 2), dict(workspace=FAKE + 4)):
        assert _matmul(**bad) == 8, bad
    assert _matmul(a_cap=api.q8_bytes(5, 40) - 1) == 7 and _matmul(b_cap=api.q8_bytes(7, 40) - 1) == 7
    assert _matmul(out_cap=5 * 7 * 4 - 1) == 7 and _matmul(stride=9, out_cap=(4 * 9 + 7) * 4 - 1) == 7
    assert _matmul(m=0, a=None, out=None) == 0 and _matmul(n=0, stride=0, b=None, out=None) == 0


def _q8_gated(**change):
    p = api.fh_q8_gated_product(FAKE, BIG, FAKE, BIG, FAKE, BIG, 5, 7, 40, FAKE, FAKE, 0, 0, 0, 0, FAKE, 7, BIG, FAKE, BIG, 0)
    for name, v in change.items():
        setattr(p, name, v)
    return LIB.fh_q8_gated(ctypes.byref(p), None)


def test_q8_gated_refusals():
    assert LIB.fh_q8_gated(None, None) == 1
    assert _q8_gated(out_dtype=2) == 2 and _q8_gated(bias_dtype=5) == 2
    for bad in (dict(m=-1), dict(n=-1), dict(k=-1), dict(stride=6), dict(k=2 ** 17), dict(m=2 ** 31), dict(stride=2 ** 31 + 1)):
        assert _q8_gated(**bad) == 11, bad
    for bad in (dict(reserved=1), dict(reserved2=1), dict(activation=3), dict(activation=-1)):
        assert _q8_gated(**bad) == 12, bad
    for name in ("x", "gate", "up", "out"):
        assert _q8_gated(**{name: None}) == 1, name
    for name in ("x", "gate", "up", "out", "gate_bias", "up_bias", "workspace"):
        assert _q8_gated(**{name: FAKE + 2}) == 8, name
    for name, rows in (("x_cap", 5), ("gate_cap", 7), ("up_cap", 7)):
        assert _q8_gated(**{name: api.q8_bytes(rows, 40) - 1}) == 7, name
    assert _q8_gated(out_cap=5 * 7 * 4 - 1) == 7
    assert _q8_gated(m=0, x=None, out=None) == 0 and _q8_gated(n=0, stride=0, gate=None, out=None) == 0


def _layer(**change):
    a = api.fh_gated_layer(50, 40, 7, 0, 0, 3, 0, FAKE, 41, FAKE, 40, FAKE, 40, FAKE, FAKE, FAKE, 7, BIG, FAKE, 7, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, BIG)
    for name, v in change.items():                               # rows of x at no multiple of 16 bytes: they are packed
        setattr(a, name, v)
    return a


@pytest.mark.parametrize("backward", [False, True])
def test_gated_refusals(backward):
    call = LIB.fh_gated_backward if backward else LIB.fh_gated

    def status(**change):
        return call(ctypes.byref(_layer(**change)), None)

    assert call(None, None) == 1 and LIB.fh_gated_workspace_bytes(None, backward) == 0
    assert status(dtype=2) == 2 and status(dtype=-1) == 2
    for bad in (dict(tokens=-1), dict(features=0), dict(hidden=0), dict(tokens=2 ** 21 + 1), dict(features=2 ** 20 + 1), dict(hidden=2 ** 20 + 1),
                dict(x_stride=39), dict(w_gate_stride=39), dict(w_up_stride=39), dict(x_stride=2 ** 31 + 1), dict(dh_stride=6) if backward else dict(h_stride=6)):
        assert status(**bad) == 11, bad
        if "dh_stride" not in bad and "h_stride" not in bad:
            assert LIB.fh_gated_workspace_bytes(ctypes.byref(_layer(**bad)), backward) == 0
    for bad in (dict(activation=3), dict(needs=4), dict(needs=-1), dict(reserved=1)):
        assert status(**bad) == 12, bad
    for name in ("x", "w_gate", "w_up", "workspace", *(("dh", "dx", "dw_gate", "dw_up") if backward else ("h",))):
        assert status(**{name: None}) == 1, name
    for name in ("x", "w_gate", "w_up", "b_gate", "b_up", "workspace", *(("dh", "dx", "dw_gate", "dw_up", "db_gate", "db_up") if backward else ("h",))):
        assert status(**{name: FAKE + 2}) == 8, name
    need = LIB.fh_gated_workspace_bytes(ctypes.byref(_layer()), backward)
    assert need > 0 and status(workspace_cap=need - 1) == 7
    if not backward:                                             # rows as the kernels want them: nothing is laid out again
        assert LIB.fh_gated_workspace_bytes(ctypes.byref(_layer(x_stride=40)), 0) == 0 == LIB.fh_gated_workspace_bytes(ctypes.byref(_layer(tokens=5)), 0)
    if backward:
        assert status(needs=0, db_gate=None, db_up=None, dh=None, workspace=None) == 0
    else:
        assert status(h_cap=50 * 7 * 4 - 1) == 7 and status(tokens=0, x=None, h=None, workspace=None) == 0


def test_the_workspace_covers_what_the_backward_call_lays_out():
    """At least the hidden width's gradients, and no less with more asked for."""
    for tokens, features, hidden, dtype in ((1, 1, 1, 0), (333, 515, 1001, 0), (8192, 768, 2048, 1), (2 ** 21, 64, 2, 1), (3, 2 ** 20, 5, 0)):
        sizes = [LIB.fh_gated_workspace_bytes(ctypes.byref(_layer(tokens=tokens, features=features, hidden=hidden, dtype=dtype, needs=needs, x_stride=features,
                                                                  w_gate_stride=features, w_up_stride=features, db_gate=None, db_up=None)), 1) for needs in (0, 1, 3)]
        assert sizes == sorted(sizes) and sizes[0] >= tokens * 2 * hidden * (4 - 2 * dtype)


def test_the_binding_refuses_host_tensors_shapes_and_names():
    x = torch.zeros(4, 40)
    m = api.Q8Matrix(torch.zeros(api.q8_bytes(4, 40), dtype=torch.uint8), 4, 40)
    for call in (lambda: api.fh_q8_quantize(x), lambda: api.fh_q8_dequantize(m), lambda: api.fh_q8_matmul(m, m), lambda: api.fh_q8_gated(m, m, m),
                 lambda: api.fh_gated(x, x, x), lambda: api.fh_gated_backward(x, x, x, x), lambda: layers.gated_linear(x, x, x),
                 lambda: layers.q8_linear(x, m), lambda: layers.GatedLinear(4, 5).freeze()):
        with pytest.raises(ValueError, match="device memory"):
            call()
    for call in (lambda: api.fh_q8_quantize(3), lambda: api.fh_gated(None, x, x)):
        with pytest.raises(TypeError, match="must be a tensor"):
            call()


def test_the_two_stored_forms_are_not_taken_for_each_other():
    q8 = api.Q8Matrix(torch.zeros(api.q8_bytes(4, 40), dtype=torch.uint8), 4, 40)
    mx = api.MxMatrix(torch.zeros(api.mx_bytes(4, 40), dtype=torch.uint8), 4, 40)
    for call in (lambda: api.fh_mx_matmul(q8, q8), lambda: api.fh_mx_dequantize(q8)):
        with pytest.raises(TypeError, match="MxMatrix"):
            call()
    for call in (lambda: api.fh_q8_matmul(mx, mx), lambda: api.fh_q8_dequantize(mx), lambda: api.fh_q8_gated(mx, mx, mx)):
        with pytest.raises(TypeError, match="Q8Matrix"):
            call()
