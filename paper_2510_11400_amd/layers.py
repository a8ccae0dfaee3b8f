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


def _rows(x: torch.Tensor) -> torch.Tensor:
    """x as a matrix of its last dimension, its rows contiguous."""
    m = x.reshape(-1, x.shape[-1])
    return m if m.stride(1) == 1 or m.shape[1] <= 1 else m.contiguous()


def _weight_gradients(dy, x_columns, weight_dtype, need_weight, need_bias, bias_dtype, dy_columns):
    dw = api.fh_mx_matmul(dy_columns, x_columns, out_dtype=weight_dtype) if need_weight else None
    db = dy.float().sum(0).to(bias_dtype) if need_bias else None
    return dw, db


class _Rounding:
    """How a layer's gradients are quantised; a step's random numbers are those of its seed."""
    __slots__ = ("mode", "seed", "tensor_id")

    def __init__(self, mode, seed, tensor_id):
        self.mode, self.seed, self.tensor_id = mode, seed, tensor_id


def _quantised_gradient(dy, rounding: _Rounding, need_input: bool, need_weight: bool):
    """(dy by rows, dy by columns), None for one that is not needed."""
    if need_input and need_weight:
        return api.fh_mx_quantize(dy, "both", rounding.mode, rounding.seed, rounding.tensor_id)
    if need_input:
        return api.fh_mx_quantize(dy, "rows", rounding.mode, rounding.seed, rounding.tensor_id), None
    if need_weight:
        return None, api.fh_mx_quantize(dy, "columns", rounding.mode, rounding.seed, rounding.tensor_id)
    return None, None


class _MxLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, rounding):
        m = _rows(x)
        need_x, need_w = ctx.needs_input_grad[0], ctx.needs_input_grad[1]
        x_rows, x_columns = api.fh_mx_quantize(m, "both") if need_w else (api.fh_mx_quantize(m, "rows"), None)
        w_rows, w_columns = api.fh_mx_quantize(weight, "both") if need_x else (api.fh_mx_quantize(weight, "rows"), None)
        y = api.fh_mx_matmul(x_rows, w_rows, bias, x.dtype)
        ctx.kept, ctx.rounding = (x_columns, w_columns), rounding
        ctx.shape, ctx.dtypes = x.shape, (weight.dtype, None if bias is None else bias.dtype)
        return y.view(*x.shape[:-1], weight.shape[0])

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        need_x, need_w, need_b = ctx.needs_input_grad[:3]
        x_columns, w_columns = ctx.kept
        g = _rows(dy)
        g_rows, g_columns = _quantised_gradient(g, ctx.rounding, need_x, need_w)
        dx = api.fh_mx_matmul(g_rows, w_columns, out_dtype=dy.dtype).view(ctx.shape) if need_x else None
        dw, db = _weight_gradients(g, x_columns, ctx.dtypes[0], need_w, need_b, ctx.dtypes[1], g_columns)
        return dx, dw, db, None


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        m = _rows(x)
        y, mean, rstd = api.fh_layer_norm(m, weight, bias, eps)
        ctx.save_for_backward(m, mean, rstd, weight)
        ctx.has_bias = bias is not None
        return y.view(x.shape)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        m, mean, rstd, weight = ctx.saved_tensors
        dx, dw, db = api.fh_layer_norm_backward(_rows(dy), m, mean, rstd, weight, sums=any(ctx.needs_input_grad[1:3]))
        return (dx.view(dy.shape) if ctx.needs_input_grad[0] else None, dw if ctx.needs_input_grad[1] else None,
                db if ctx.needs_input_grad[2] else None, None)


class _LayerNormMxLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, norm_weight, norm_bias, weight, bias, eps, rounding):
        m = _rows(x)
        need_norm, need_w = any(ctx.needs_input_grad[:3]), ctx.needs_input_grad[3]
        h, mean, rstd = api.fh_layer_norm_mx(m, norm_weight, norm_bias, eps, "both" if need_w else "rows")
        h_rows, h_columns = h if need_w else (h, None)
        w_rows, w_columns = api.fh_mx_quantize(weight, "both") if need_norm else (api.fh_mx_quantize(weight, "rows"), None)
        y = api.fh_mx_matmul(h_rows, w_rows, bias, x.dtype)
        ctx.kept, ctx.rounding, ctx.shape = (h_columns, w_columns), rounding, x.shape
        ctx.dtypes = weight.dtype, None if bias is None else bias.dtype
        if need_norm:
            ctx.save_for_backward(m, mean, rstd, norm_weight)
        return y.view(*x.shape[:-1], weight.shape[0])

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        need_norm, (need_w, need_b) = any(ctx.needs_input_grad[:3]), ctx.needs_input_grad[3:5]
        h_columns, w_columns = ctx.kept
        g = _rows(dy)
        g_rows, g_columns = _quantised_gradient(g, ctx.rounding, need_norm, need_w)
        dw, db = _weight_gradients(g, h_columns, ctx.dtypes[0], need_w, need_b, ctx.dtypes[1], g_columns)
        dx = d_norm_weight = d_norm_bias = None
        if need_norm:
            m, mean, rstd, norm_weight = ctx.saved_tensors
            dh = api.fh_mx_matmul(g_rows, w_columns, out_dtype=dy.dtype)
            dx, d_norm_weight, d_norm_bias = api.fh_layer_norm_backward(dh, m, mean, rstd, norm_weight, dx=dh,
                                                                        sums=any(ctx.needs_input_grad[1:3]))
            dx = dx.view(ctx.shape) if ctx.needs_input_grad[0] else None
        return (dx, d_norm_weight if ctx.needs_input_grad[1] else None, d_norm_bias if ctx.needs_input_grad[2] else None, dw, db, None, None)


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5) -> torch.Tensor:
    """Layer norm over the last dimension, differentiable.  x is saved as it is: under hooks.SavedActivations it is stored
    compressed, like any activation that autograd saves."""
    return _LayerNorm.apply(x, weight, bias, eps)


def mx_linear(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, rounding="nearest", seed: int = 0,
              tensor_id: int = 0) -> torch.Tensor:
    """x W^T + bias with all three products of a training step in microscaled 4-bit form.  rounding, seed and tensor_id
    are those of the gradient's quantisation; activations and weights are rounded to the nearest."""
    return _MxLinear.apply(x, weight, bias, _Rounding(rounding, seed, tensor_id))


def layer_norm_mx_linear(x: torch.Tensor, norm_weight: Optional[torch.Tensor], norm_bias: Optional[torch.Tensor], weight: torch.Tensor,
                         bias: Optional[torch.Tensor] = None, eps: float = 1e-5, rounding="nearest", seed: int = 0,
                         tensor_id: int = 0) -> torch.Tensor:
    """mx_linear(layer_norm(x)) without the norm's output ever being written but as codes."""
    return _LayerNormMxLinear.apply(x, norm_weight, norm_bias, weight, bias, eps, _Rounding(rounding, seed, tensor_id))


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
    of forward passes so far, the tensor id `tensor_id`.  A frozen layer runs two kernels for any number of tokens."""

    def __init__(self, features: int, out_features: int, bias: bool = True, eps: float = 1e-5, rounding="nearest", seed: int = 0,
                 tensor_id: int = 0, device=None, dtype=None):
        super().__init__()
        self.norm = LayerNorm(features, eps, device=device, dtype=dtype)
        self.linear = torch.nn.Linear(features, out_features, bias=bias, device=device, dtype=dtype)
        self.rounding, self.seed, self.tensor_id, self.steps = rounding, seed, tensor_id, 0
        self._stored: Optional[api.MxMatrix] = None

    def freeze(self) -> "LayerNormMxLinear":
        """Store the weights in 4-bit blocks; from here on forward() uses these and gives no gradients.  Call it again after
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
        with torch.no_grad():
            h, _, _ = api.fh_layer_norm_mx(_rows(x), self.norm.weight, self.norm.bias, self.norm.eps, "rows")
            y = api.fh_mx_matmul(h, self._stored, self.linear.bias, x.dtype)
        return y.view(*x.shape[:-1], self._stored.rows)
