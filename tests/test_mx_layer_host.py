"""The linear layer's calls without a GPU: what they ask for and refuse ahead of any launch."""
from __future__ import annotations

import ctypes

import pytest
import torch

from paper_2510_11400_amd import api, layers

FAKE = 0x10000  # an aligned non-NULL address; never dereferenced because validation fails first
LIB = api.raw_library()
BF16 = 1


def _layer(**change):
    a = api.fh_mx_layer(tokens=100, features=300, out_features=70, dtype=BF16, p_dtype=0, norm=1, needs=3, rounding=0, eps=1e-5, x=FAKE, x_stride=300,
                        norm_weight=FAKE, norm_bias=FAKE, weight=FAKE, weight_stride=300, bias=FAKE, y=FAKE, dy=FAKE, dy_stride=70, dx=FAKE, dweight=FAKE,
                        dnorm_weight=FAKE, dnorm_bias=FAKE, kept=FAKE, kept_cap=1 << 40, scratch=FAKE, scratch_cap=1 << 40)
    for name, v in change.items():
        assert hasattr(a, name)
        setattr(a, name, v)
    return a


def _sizes(**change):
    """(status, kept, forward scratch, backward scratch)"""
    out = [ctypes.c_size_t(0) for _ in range(3)]
    a = _layer(**change)
    return (LIB.fh_mx_layer_sizes(ctypes.byref(a), *(ctypes.byref(v) for v in out)), *(v.value for v in out))


def test_a_wide_gradient_asks_for_room():
    """The fp32 gradient lies in the scratch of the backward call, where there is one that would be rounded otherwise."""
    status, kept, forward, backward = _sizes()
    assert status == 0 and kept == LIB.fh_mx_layer_kept_bytes(100, 300, 70) and max(forward, backward) == LIB.fh_mx_layer_scratch_bytes(100, 300, 70)
    status, kept2, forward2, wide = _sizes(wide_gradient=1)
    assert (status, kept2, forward2) == (0, kept, forward) and wide >= api.mx_bytes(100, 70) + 4 * 100 * 300 and wide > backward
    for change in (dict(norm=0), dict(needs=2), dict(dtype=0)):
        assert _sizes(wide_gradient=1, **change)[3] == _sizes(**change)[3]
    assert LIB.fh_mx_layer_backward(ctypes.byref(_layer(wide_gradient=1, scratch_cap=wide - 1)), None) == 7


@pytest.mark.parametrize("change, status", [(dict(wide_gradient=2), 12), (dict(wide_gradient=-1), 12), (dict(tokens=-1), 11), (dict(dtype=7), 2), (dict(norm=3), 12)])
def test_sizes_of_a_layer_that_is_refused(change, status):
    assert _sizes(**change) == (status, 0, 0, 0)
    for call in (LIB.fh_mx_layer_forward, LIB.fh_mx_layer_backward):
        assert call(ctypes.byref(_layer(**change)), None) == status


def test_sizes_want_somewhere_to_go():
    one = ctypes.byref(ctypes.c_size_t(0))
    a = ctypes.byref(_layer())
    assert LIB.fh_mx_layer_sizes(None, one, one, one) == 1
    assert LIB.fh_mx_layer_sizes(a, None, one, one) == 1 and LIB.fh_mx_layer_sizes(a, one, None, one) == 1 and LIB.fh_mx_layer_sizes(a, one, one, None) == 1


@pytest.mark.parametrize("before, again", [(True, False), (False, True)])
def test_the_norms_weight_is_given_again(before, again):
    """Left out, the gradients would be those of a weight of ones."""
    x, w, nw = torch.zeros(4, 40), torch.zeros(7, 40), torch.ones(40)
    layer = api.MxLayer(x, w, norm=True, norm_weight=nw if before else None)
    layer.shape, layer.dtype = torch.Size((4, 7)), torch.float32                # as a forward call leaves them
    layer.kept, layer.features, layer.p_dtype, layer.kept_for = None, 40, torch.float32, 3
    with pytest.raises(ValueError, match="norm_weight"):
        layer.backward(torch.zeros(4, 7), x, nw if again else None)
    with pytest.raises(ValueError, match="device memory"):                      # alike: on to the call itself, which wants device tensors
        layer.backward(torch.zeros(4, 7), x, nw if before else None)


@pytest.mark.parametrize("which", range(5))
def test_tangents_are_refused(which):
    """A tensor with a tangent requires no gradient, and the kernels know nothing of it: y without one would be a derivative of zero."""
    tensors = [torch.randn(s) for s in ((6, 40), (40,), (40,), (7, 40), (7,))]
    with torch.autograd.forward_ad.dual_level():
        dual = [torch.autograd.forward_ad.make_dual(t, torch.ones_like(t)) if i == which else t for i, t in enumerate(tensors)]
        with pytest.raises(NotImplementedError, match="tangent"):
            layers.layer_norm_mx_linear(*dual)
        if which in (0, 3, 4):
            with pytest.raises(NotImplementedError, match="tangent"):
                layers.mx_linear(dual[0], dual[3], dual[4])
        frozen = layers.LayerNormMxLinear(40, 7)
        frozen._stored = api.MxMatrix(torch.zeros(api.mx_bytes(7, 40), dtype=torch.uint8), 7, 40)
        if which == 0:
            with pytest.raises(NotImplementedError, match="tangent"):
                frozen(dual[0])
    with pytest.raises(ValueError, match="device memory"):       # without one: on to the call itself, which wants device tensors
        layers.layer_norm_mx_linear(*tensors)
    with pytest.raises(ValueError, match="device memory"):
        frozen(tensors[0])


def test_only_what_is_needed_is_kept():
    """With kept_for: x by columns for the weight's gradient, W by columns for the input's, statistics with a norm; without, room for all."""
    whole = lambda n: -(-n // 256) * 256  # noqa: E731
    stats, x, w = 2 * whole(400), whole(api.mx_bytes(300, 100)), whole(api.mx_bytes(300, 70))
    assert [_sizes(needs=n, kept_for=n)[1] for n in (1, 2, 3)] == [stats + w, stats + x, stats + x + w]
    assert [_sizes(needs=n, kept_for=n, norm=0)[1] for n in (1, 2, 3)] == [w, x, x + w]
    assert [_sizes(needs=n, kept_for=3)[1] for n in (1, 2)] == [stats + x + w] * 2
    assert [_sizes(needs=n)[1] for n in (1, 2, 3)] == [LIB.fh_mx_layer_kept_bytes(100, 300, 70)] * 3 == [stats + x + w] * 3
    assert _sizes(needs=0)[:2] == (0, 0) and _sizes(needs=0, norm=0)[:2] == (0, 0)
    for n in (1, 2):
        assert _sizes(needs=3, kept_for=n)[0] == 12 and _sizes(needs=3 - n, kept_for=n)[0] == 12
        for call in (LIB.fh_mx_layer_forward, LIB.fh_mx_layer_backward):
            assert call(ctypes.byref(_layer(needs=n, kept_for=n, kept_cap=_sizes(needs=n, kept_for=n)[1] - 1)), None) == 7
            assert call(ctypes.byref(_layer(needs=n, kept_for=n, kept=None)), None) == 1
    assert _sizes(kept_for=4)[0] == 12 and _sizes(kept_for=-1)[0] == 12
