"""Embeddings: the rows of a table that class labels, code maps or tokens name, as channels-last input of the layers, and the
gradient of the table.  Forward and backward pass are one native call each (xconv_embed_fwd / xconv_embed_bwd); the gradient adds up the
places of every row in an order that depends on the indices alone, so it is the same bits every time."""
import math

import torch

from .layer import _DTYPE, _glue, _raw_stream


def _check_values(x):
    if not x.is_cuda:
        raise RuntimeError("embedding: runs on the GPU only (values on %s)" % x.device)
    if x.dtype not in _DTYPE:
        raise RuntimeError("embedding: storage type %s is not supported (float32, bfloat16, float16)" % x.dtype)


def embedding_forward(indices, weight, scale=1.0):
    """scale * weight[indices], [indices' shape, C]; an index outside the table gives a row of NaN."""
    _check_values(weight)
    return _glue().embed_forward(indices, weight, scale, _raw_stream(weight))


def embedding_backward(dy, indices, rows, scale=1.0, padding_idx=None, dtype=None):
    """The gradient [rows, C] of the table from that of the output; `dtype` float32 or the type of dy (None).  The row padding_idx
    (a negative one counts from the end) gets none, nor does an index outside the table give any."""
    _check_values(dy)
    if dtype not in (None, torch.float32, dy.dtype):
        raise RuntimeError("embedding: the gradient of the table is float32 or of the output's type, not %s" % dtype)
    # for the library -1 is none, and what is still below it is refused there
    row = -1 if padding_idx is None else padding_idx if padding_idx >= 0 else padding_idx + rows if padding_idx >= -rows else -2
    return _glue().embed_backward(dy, indices, rows, scale, row, dtype == torch.float32, _raw_stream(dy))


class _EmbeddingFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, indices, weight, scale, padding_idx):
        ctx.save_for_backward(indices)
        ctx.rows, ctx.scale, ctx.padding_idx, ctx.dtype = weight.shape[0], scale, padding_idx, weight.dtype
        return embedding_forward(indices, weight, scale)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        (indices,) = ctx.saved_tensors
        dw = embedding_backward(dy.to(ctx.dtype), indices, ctx.rows, ctx.scale, ctx.padding_idx) if ctx.needs_input_grad[1] else None
        return None, dw, None, None


def _row(padding_idx, rows):
    """torch's convention: negative ones count from the end"""
    if padding_idx is None:
        return None
    if not -rows <= padding_idx < rows:
        raise ValueError("embedding: padding_idx must be a row of the table")
    return padding_idx % rows


def embedding(indices, weight, scale=1.0, padding_idx=None, axis=-1):
    """scale * weight[indices], differentiable (once) in weight, with the channels at `axis`: -1, or 1 ([B, C, ...], channels-last in
    memory as the layers take it)."""
    if axis not in (-1, 1):
        raise ValueError("embedding: axis must be -1 or 1")
    if axis == 1 and indices.dim() < 1:
        raise ValueError("embedding: channels at axis 1 need a batch axis")
    y = _EmbeddingFunction.apply(indices, weight, scale, _row(padding_idx, weight.shape[0]))
    return y if axis == -1 else y.movedim(-1, 1)


class XEmbedding(torch.nn.Module):
    """torch.nn.Embedding of `rows` rows (same parameter and padding_idx) whose output is multiplied by `scale` and has its channels at
    `axis` (-1, or 1 for code maps [B, H, W] in front of convolutions)."""

    def __init__(self, rows, channels, scale=1.0, padding_idx=None, axis=-1, device=None, dtype=None):
        super().__init__()
        if int(rows) < 1 or int(channels) < 1:
            raise ValueError("XEmbedding: at least one row and one channel")
        if axis not in (-1, 1):
            raise ValueError("XEmbedding: axis must be -1 or 1")
        if not math.isfinite(scale):
            raise ValueError("XEmbedding: scale must be finite")
        self.rows, self.channels, self.scale, self.axis = int(rows), int(channels), float(scale), axis
        self.padding_idx = _row(padding_idx, self.rows)
        self.weight = torch.nn.Parameter(torch.empty(self.rows, self.channels, device=device, dtype=dtype))
        with torch.no_grad():
            self.weight.normal_()
            if self.padding_idx is not None:
                self.weight[self.padding_idx].zero_()

    def forward(self, indices):
        return embedding(indices, self.weight, self.scale, self.padding_idx, self.axis)

    def extra_repr(self):
        return "%d, %d, scale=%g, axis=%d" % (self.rows, self.channels, self.scale, self.axis)


__all__ = ["XEmbedding", "embedding", "embedding_backward", "embedding_forward"]
