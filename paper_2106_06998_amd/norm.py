"""Layer normalisation over the channels of every position: what stands between the convolutions of a network
that normalises without batch statistics.  Forward and backward pass are one native call each on the library's
kernels (xconv_layernorm_fwd / xconv_layernorm_bwd); sums are fp32 whatever the storage type.

Channels are the last axis (rows, channels-last activations) or axis 1 ([B, C, H, W] planes or volumes; a
channels-last tensor is read as it lies)."""
import torch

from .layer import _DTYPE, _glue, _raw_stream


def _check_input(x):
    if not x.is_cuda:
        raise RuntimeError("layer_norm: runs on the GPU only (input on %s)" % x.device)
    if x.dtype not in _DTYPE:
        raise RuntimeError("layer_norm: storage type %s is not supported (float32, bfloat16, float16)" % x.dtype)


def layer_norm_forward(x, weight=None, bias=None, eps=1e-5, axis=-1):
    """(y, mean, rstd) of `x` normalised over `axis` (the last or 1); weight and bias are [C] in float32 or the
    type of x, None for ones and zeros.  mean and rstd are float32 with the shape of x without the axis."""
    _check_input(x)
    return _glue().norm_forward(x, weight, bias, eps, axis, _raw_stream(x))


def layer_norm_backward(dy, x, mean, rstd, weight=None, axis=-1, need=(True, True, True), param_dtype=None):
    """(dx, dweight, dbias) from the forward pass's input and statistics; `need` says which are wanted (None for the
    others).  dweight and dbias are of the weight's type; without a weight of `param_dtype`, float32 or the type of x (None)."""
    _check_input(x)
    if weight is not None or param_dtype is None:
        param_dtype = x.dtype if weight is None else weight.dtype
    if param_dtype not in (torch.float32, x.dtype):
        raise RuntimeError("layer_norm: parameters are float32 or of the input's type, not %s" % param_dtype)
    return _glue().norm_backward(dy, x, mean, rstd, weight, axis, need[0], need[1], need[2], param_dtype == torch.float32, _raw_stream(x))


class _LayerNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, axis):
        y, mean, rstd = layer_norm_forward(x, weight, bias, eps, axis)
        ctx.save_for_backward(x, mean, rstd, weight)
        ctx.axis, ctx.bias_dtype = axis, None if bias is None else bias.dtype
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, mean, rstd, weight = ctx.saved_tensors
        dx, dw, db = layer_norm_backward(dy, x, mean, rstd, weight, ctx.axis, ctx.needs_input_grad[:3], ctx.bias_dtype)
        return dx, dw, db, None, None


def layer_norm(x, weight=None, bias=None, eps=1e-5, axis=-1):
    """layer_norm_forward's y, differentiable (once) in x, weight and bias."""
    return _LayerNormFunction.apply(x, weight, bias, eps, axis)


class XLayerNorm(torch.nn.Module):
    """Layer normalisation over `channels` channels at `axis`: -1 for rows and channels-last layouts, as
    torch.nn.LayerNorm over the last axis (same parameters), or 1 for the activations of convolutions."""

    def __init__(self, channels, eps=1e-5, axis=-1, elementwise_affine=True, bias=True, device=None, dtype=None):
        super().__init__()
        if int(channels) < 1:
            raise ValueError("XLayerNorm: at least one channel")
        if axis not in (-1, 1):
            raise ValueError("XLayerNorm: axis must be -1 or 1")
        if not eps >= 0:
            raise ValueError("XLayerNorm: eps must not be negative")
        self.channels, self.eps, self.axis = int(channels), float(eps), axis
        kw = {"device": device, "dtype": dtype}
        self.weight = torch.nn.Parameter(torch.ones(self.channels, **kw)) if elementwise_affine else None
        self.bias = torch.nn.Parameter(torch.zeros(self.channels, **kw)) if elementwise_affine and bias else None

    def forward(self, x):
        if x.dim() < (1 if self.axis == -1 else 2) or x.shape[self.axis] != self.channels:
            raise RuntimeError("XLayerNorm: expected %d channels at axis %d, got an input of %s" % (self.channels, self.axis, tuple(x.shape)))
        return layer_norm(x, self.weight, self.bias, self.eps, self.axis)

    def extra_repr(self):
        return "%d, eps=%g, axis=%d" % (self.channels, self.eps, self.axis)


__all__ = ["XLayerNorm", "layer_norm", "layer_norm_backward", "layer_norm_forward"]
