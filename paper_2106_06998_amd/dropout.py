"""Dropout whose mask is never stored: every value of it is drawn from a seed where it is applied (xconv_dropout), as the layers
draw their probing vectors, so that the backward pass needs the seed alone.

A value is dropped with probability p, taken to the nearest multiple of 2^-16, and the others are divided by the probability that
is left; places count in memory order.  A dropped value is zero also where it was an infinity or a NaN."""
import torch

from . import binding as xb
from .layer import _DTYPE, _glue, _raw_stream


def _rate(p, who="dropout"):
    """values of 65536 that are dropped"""
    if not 0 <= p <= 1:
        raise ValueError("%s: p must lie in [0, 1]" % who)
    return int(65536 * p + 0.5)


def _seed(seed):
    """any 64 bits, as a signed number"""
    seed &= 0xFFFFFFFFFFFFFFFF
    return seed - (1 << 64) if seed >> 63 else seed


def _check_input(x):
    if not x.is_cuda:
        raise RuntimeError("dropout: runs on the GPU only (input on %s)" % x.device)
    if x.dtype not in _DTYPE:
        raise RuntimeError("dropout: storage type %s is not supported (float32, bfloat16, float16)" % x.dtype)


def dropout_forward(x, p, seed, step=None):
    """`x` with the mask of `seed` applied, in the memory order of x (that of a contiguous copy where x has gaps).  step: an int64
    tensor of one value on the device that is added to the seed when the kernel runs; calls that share one take seeds that are further
    apart than it goes (random ones), as the mask goes by the sum."""
    _check_input(x)
    return _glue().dropout(x, _rate(p), _seed(seed), step, None, _raw_stream(x))


def dropout_backward(dy, p, seed, step=None):
    """The gradient of dropout_forward's input from that of its output, which lies in the same memory order."""
    return dropout_forward(dy, p, seed, step)


class _DropoutFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, p, seed, step):
        y = dropout_forward(x, p, seed, step)
        ctx.save_for_backward(step)                                            # (a step that changes before the backward pass is noticed)
        ctx.meta = (tuple(y.shape), y.stride(), xb.DTYPES[_DTYPE[y.dtype]])
        ctx.p, ctx.seed = p, seed
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        (step,) = ctx.saved_tensors
        _check_input(dy)
        return _glue().dropout(dy, _rate(ctx.p), _seed(ctx.seed), step, ctx.meta, _raw_stream(dy)), None, None, None


def dropout(x, p, seed, step=None):
    """dropout_forward, differentiable (once) in x."""
    return _DropoutFunction.apply(x, p, seed, step)


class _Draws:
    """The seeds of a module: another one for every forward pass, drawn from torch's default CPU generator (and `base_seed`).  So they follow
    torch.manual_seed and a saved state of the generator, torch.utils.checkpoint draws the same ones for the pass that it runs again, and
    the masks of processes are unlike where their generators (or base seeds) are.  A captured graph keeps the seed that it was captured
    with, so there a `step` is expected, which the program advances between replays.  (As with any module, a backward pass is captured
    while no eager graph of the same parameters is kept: torch's engine ends the process otherwise.)"""

    def _next_seed(self, x):
        if self.step is None and x.is_cuda and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("%s: a captured graph would apply one mask on every replay; give the module a step tensor and advance it" % type(self).__name__)
        self.last_seed = _glue().draw_seed(_seed(self.base_seed))
        return self.last_seed


class XDropout(torch.nn.Module, _Draws):
    """torch.nn.Dropout that keeps a seed in place of its mask, drawn from torch's default CPU generator in every training forward call
    (`last_seed` is the latest).  step: an int64 tensor of one value on the device, added to the seed (for captured graphs; it must not
    change between the forward and the backward pass)."""

    def __init__(self, p=0.5, base_seed=0, step=None):
        super().__init__()
        _rate(p, "XDropout")
        self.p, self.base_seed, self.step, self.last_seed = float(p), int(base_seed), step, None

    def forward(self, x):
        if not self.training or _rate(self.p) == 0:
            return x
        return dropout(x, self.p, self._next_seed(x), self.step)

    def extra_repr(self):
        return "p=%g" % self.p


__all__ = ["XDropout", "dropout", "dropout_backward", "dropout_forward"]
