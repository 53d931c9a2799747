"""Normalisation over the channels of every position: what stands between the convolutions of a network
that normalises without batch statistics.  Forward and backward pass are one native call each on the library's
kernels (xconv_layernorm_fwd / xconv_layernorm_bwd, xconv_rmsnorm_fwd / xconv_rmsnorm_bwd); sums are fp32 whatever the storage type.

layer_norm takes the mean out and divides by the deviation; rms_norm divides by the root of the mean square, and adds the
residual stream to the (dropped out) branch on the way.  rms_norm_8bit is the form for serving whose output is 8 bits and a scale.

Channels are the last axis (rows, channels-last activations) or axis 1 ([B, C, H, W] planes or volumes; a
channels-last tensor is read as it lies)."""
import torch

from .dropout import _Draws, _rate, _seed
from .layer import _DTYPE, _glue, _raw_stream


def _check_input(x, who="layer_norm"):
    if not x.is_cuda:
        raise RuntimeError("%s: runs on the GPU only (input on %s)" % (who, x.device))
    if x.dtype not in _DTYPE:
        raise RuntimeError("%s: storage type %s is not supported (float32, bfloat16, float16)" % (who, x.dtype))


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


def rms_norm_forward(x, weight=None, residual=None, eps=1e-6, axis=-1, p=0.0, seed=0, step=None):
    """(y, h, rstd): h = residual + dropout(x), y = h rstd weight with rstd = 1/sqrt(mean of h^2 over `axis` + eps) (the last axis or 1).
    weight is [C] in float32 or the type of x, None for ones; residual is of the shape and type of x.  h is x itself without a residual and
    dropout; rstd is float32 with the shape of x without the axis.  p, seed, step: as of dropout_forward."""
    _check_input(x, "rms_norm")
    y, h, rstd = _glue().rms_forward(x, weight, residual, eps, axis, _rate(p, "rms_norm"), _seed(seed), step, _raw_stream(x))
    return y, x if h is None else h, rstd


def rms_norm_backward(dy, h, rstd, weight=None, dh=None, axis=-1, p=0.0, seed=0, step=None, need=(True, True, True), param_dtype=None):
    """(dx, dresidual, dweight) from the gradients of y and of h (None: zeros) and the forward pass's h and rstd; `need` says which are
    wanted (None for the others).  Without dropout dx and dresidual are one tensor.  dweight is of the weight's type; without a weight of
    `param_dtype`, float32 or the type of h (None)."""
    _check_input(h, "rms_norm")
    if weight is not None or param_dtype is None:
        param_dtype = h.dtype if weight is None else weight.dtype
    if param_dtype not in (torch.float32, h.dtype):
        raise RuntimeError("rms_norm: parameters are float32 or of the input's type, not %s" % param_dtype)
    return _glue().rms_backward(dy, h, rstd, weight, dh, axis, _rate(p, "rms_norm"), _seed(seed), need[0], need[1], need[2], param_dtype == torch.float32,
                                step, _raw_stream(h))


_TYPE_8BIT = {torch.float8_e4m3fn: 0, torch.int8: 1}


def rms_norm_8bit(x, weight=None, residual=None, eps=1e-6, axis=-1, dtype=torch.float8_e4m3fn):
    """(q, scale, h): rms_norm_forward's y as q * scale with one float32 scale a position and q of `dtype` (torch.float8_e4m3fn or torch.int8);
    the largest magnitude of a position is 448 (127) times its scale.  Not differentiable."""
    _check_input(x, "rms_norm_8bit")
    if dtype not in _TYPE_8BIT:
        raise RuntimeError("rms_norm_8bit: the output is torch.float8_e4m3fn or torch.int8, not %s" % dtype)
    q, scale, h = _glue().rms_forward_8bit(x, weight, residual, eps, axis, _TYPE_8BIT[dtype], _raw_stream(x))
    return q, scale, x if h is None else h


class _RMSNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, eps, axis, p, seed, step):
        y, h, rstd = rms_norm_forward(x, weight, residual, eps, axis, p, seed, step)
        ctx.save_for_backward(h, rstd, weight, step)
        ctx.axis, ctx.p, ctx.seed, ctx.streams = axis, p, seed, residual is not None
        ctx.set_materialize_grads(False)
        return (y, h) if ctx.streams else y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dh=None):
        h, rstd, weight, step = ctx.saved_tensors
        need = (ctx.needs_input_grad[0], ctx.needs_input_grad[2], weight is not None and ctx.needs_input_grad[1])
        if dy is None and dh is None:
            return (None,) * 8
        if dy is None:                  # only h is used
            dy = torch.zeros_like(h)
        dx, dresidual, dw = rms_norm_backward(dy, h, rstd, weight, dh, ctx.axis, ctx.p, ctx.seed, step, need)
        return dx, dw, dresidual, None, None, None, None, None


def rms_norm(x, weight=None, residual=None, eps=1e-6, axis=-1, p=0.0, seed=0, step=None):
    """rms_norm_forward's y, or (y, h) with a residual, differentiable (once) in x, weight and residual."""
    return _RMSNormFunction.apply(x, weight, residual, eps, axis, p, seed, step)


class XRMSNorm(torch.nn.Module, _Draws):
    """Root-mean-square norm over `channels` channels at `axis` (-1 or 1 as of XLayerNorm; parameters as torch.nn.RMSNorm).  Called with a
    residual it returns (y, h): h = residual + x goes on as the residual stream, y into the next branch.  p: dropout of x in training,
    from a seed that every forward call draws (`last_seed`; generator, step and captured graphs: as of XDropout)."""

    def __init__(self, channels, eps=1e-6, axis=-1, elementwise_affine=True, p=0.0, base_seed=0, step=None, device=None, dtype=None):
        super().__init__()
        if int(channels) < 1:
            raise ValueError("XRMSNorm: at least one channel")
        if axis not in (-1, 1):
            raise ValueError("XRMSNorm: axis must be -1 or 1")
        if not eps >= 0:
            raise ValueError("XRMSNorm: eps must not be negative")
        _rate(p, "XRMSNorm")
        self.channels, self.eps, self.axis, self.p = int(channels), float(eps), axis, float(p)
        self.base_seed, self.step, self.last_seed = int(base_seed), step, None
        self.weight = torch.nn.Parameter(torch.ones(self.channels, device=device, dtype=dtype)) if elementwise_affine else None

    def forward(self, x, residual=None):
        if x.dim() < (1 if self.axis == -1 else 2) or x.shape[self.axis] != self.channels:
            raise RuntimeError("XRMSNorm: expected %d channels at axis %d, got an input of %s" % (self.channels, self.axis, tuple(x.shape)))
        drops = self.training and _rate(self.p) > 0
        return rms_norm(x, self.weight, residual, self.eps, self.axis, self.p if drops else 0.0, self._next_seed(x) if drops else 0, self.step if drops else None)

    def extra_repr(self):
        return "%d, eps=%g, axis=%d, p=%g" % (self.channels, self.eps, self.axis, self.p)


__all__ = ["XLayerNorm", "XRMSNorm", "layer_norm", "layer_norm_backward", "layer_norm_forward", "rms_norm", "rms_norm_8bit", "rms_norm_backward",
           "rms_norm_forward"]
