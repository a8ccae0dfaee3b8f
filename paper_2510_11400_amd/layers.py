"""Layers whose saved activations are stored in microscaled 4-bit form and used as they are stored.

`SavedActivations` (hooks.py) compresses what autograd saves and restores it before the backward pass reads it
(FedHybrid Section 3: compress in the forward pass, decompress during backpropagation).  The layers here go one step
further for matrix products: the input of a linear layer is kept in 4-bit blocks along the tokens, which is an operand of
the weight's gradient as it is, so nothing is restored.  Behind a layer norm it never exists in 16 bits at all.

    y  = x W^T + b      x and W by rows                      (forward)
    dx = dy W           dy by rows, W by columns             (backward)
    dW = dy^T x         dy by columns, x by columns (the saved form)

Matrix products are of 4-bit values with binary32 sums; parameters and their gradients keep their own dtype.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import api
from .api import _binding


def _rows(x: torch.Tensor) -> torch.Tensor:
    """x as a matrix of its last dimension, its rows contiguous and apart (an expanded gradient's are not)."""
    m = x if x.dim() == 2 else x.reshape(-1, x.shape[-1])
    stride, step = m.stride()
    return m if step == 1 and stride >= m.shape[1] else m.contiguous()


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        m = _rows(x)
        y, mean, rstd = api.fh_layer_norm(m, weight, bias, eps)
        # the statistics as bytes: hooks.SavedActivations would quantise vectors of fp32 from 4096 rows on, and an rstd that is small beside its
        # group's others would be off by any factor
        ctx.sums_dtype = None if weight is not None or bias is None else bias.dtype
        ctx.save_for_backward(m, mean.view(torch.uint8), rstd.view(torch.uint8), weight)
        return y.view(x.shape)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        m, mean, rstd, weight = ctx.saved_tensors
        mean, rstd = mean.view(torch.float32), rstd.view(torch.float32)
        dx, dw, db = api.fh_layer_norm_backward(_rows(dy), m, mean, rstd, weight, sums=any(ctx.needs_input_grad[1:3]),
                                                sums_dtype=ctx.sums_dtype)
        return (dx.view(dy.shape) if ctx.needs_input_grad[0] else None, dw if ctx.needs_input_grad[1] else None,
                db if ctx.needs_input_grad[2] else None, None)


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5) -> torch.Tensor:
    """Layer norm over the last dimension, differentiable.  x is saved as it is: under hooks.SavedActivations it is stored
    compressed, like any activation that autograd saves; the rows' statistics stay exact."""
    return _LayerNorm.apply(x, weight, bias, eps)


def mx_linear(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, rounding="nearest", seed: int = 0,
              tensor_id: int = 0) -> torch.Tensor:
    """x W^T + bias with all three products of a training step in microscaled 4-bit form.  rounding, seed and tensor_id
    are those of the gradient's quantisation; activations and weights are rounded to the nearest."""
    return _binding.mx_linear(x, None, None, weight, bias, None, rounding, seed, tensor_id)


def layer_norm_mx_linear(x: torch.Tensor, norm_weight: Optional[torch.Tensor], norm_bias: Optional[torch.Tensor], weight: torch.Tensor,
                         bias: Optional[torch.Tensor] = None, eps: float = 1e-5, rounding="nearest", seed: int = 0,
                         tensor_id: int = 0) -> torch.Tensor:
    """mx_linear(layer_norm(x)) without the norm's output ever being written but as codes.  x is saved as autograd saves it
    (hooks.SavedActivations compresses it); the product's operands are kept in 4-bit form.  The parameters are of one dtype.
    Backward, the norm takes its output's gradient in fp32."""
    return _binding.mx_linear(x, norm_weight, norm_bias, weight, bias, eps, rounding, seed, tensor_id)


class LayerNorm(torch.nn.Module):
    """Layer norm over the last dimension."""

    def __init__(self, features: int, eps: float = 1e-5, affine: bool = True, device=None, dtype=None):
        super().__init__()
        self.eps = eps
        self.weight = torch.nn.Parameter(torch.ones(features, device=device, dtype=dtype)) if affine else None
        self.bias = torch.nn.Parameter(torch.zeros(features, device=device, dtype=dtype)) if affine else None

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return layer_norm(x, self.weight, self.bias, self.eps)


class LayerNormMxLinear(torch.nn.Module):
    """A layer norm and the linear layer behind it, trained in 4-bit blocks; `freeze()` stores the weights once for serving.

    With stochastic rounding of the gradients every step draws its own random numbers: the seed is `seed` plus the number
    of forward passes so far, the tensor id `tensor_id` (a graph replays the numbers of its capture).  A frozen layer runs two kernels for any number of tokens."""

    def __init__(self, features: int, out_features: int, bias: bool = True, eps: float = 1e-5, rounding="nearest", seed: int = 0,
                 tensor_id: int = 0, device=None, dtype=None):
        super().__init__()
        self.norm = LayerNorm(features, eps, device=device, dtype=dtype)
        self.linear = torch.nn.Linear(features, out_features, bias=bias, device=device, dtype=dtype)
        self.rounding, self.seed, self.tensor_id, self.steps = rounding, seed, tensor_id, 0
        self._stored: Optional[api.MxMatrix] = None

    def freeze(self) -> "LayerNormMxLinear":
        """Store the weights in 4-bit blocks; from here on forward() uses these and gives no gradients (tangents are refused).  Call it again after
        the weights have changed, `thaw()` to train on."""
        self._stored = api.fh_mx_quantize(self.linear.weight.detach(), "rows")
        return self

    def thaw(self) -> "LayerNormMxLinear":
        self._stored = None
        return self

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        if self._stored is None:
            seed, self.steps = self.seed + self.steps, self.steps + 1
            return layer_norm_mx_linear(x, self.norm.weight, self.norm.bias, self.linear.weight, self.linear.bias, self.norm.eps,
                                        self.rounding, seed, self.tensor_id)
        norm_weight, norm_bias, bias = self.norm.weight, self.norm.bias, self.linear.bias
        _binding.refuse_tangents(x, norm_weight, norm_bias, bias)
        with torch.no_grad():
            h, _, _ = api.fh_layer_norm_mx(_rows(x), norm_weight, norm_bias, self.norm.eps, "rows")
            y = api.fh_mx_matmul(h, self._stored, bias, x.dtype)
        return y.view(*x.shape[:-1], self._stored.rows)
