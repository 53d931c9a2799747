"""Dropout masks, the root-mean-square norm and embeddings in 64 bits, from their definitions, with bounds of what fp32 arithmetic and
one rounding may differ by.  u = 2^-24 is half a step of fp32, half(t) that of a storage type."""
import numpy as np
import torch

U = 2.0 ** -24
SIZES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LEAST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}     # smallest subnormal number


def half(dtype):
    return torch.finfo(dtype).eps / 2


def rounding(value, dtype):
    """what one rounding to `dtype` may change"""
    return value.abs() * half(dtype) + LEAST[dtype]


def fin(z):
    mask = (1 << 64) - 1
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & mask
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & mask
    return z ^ (z >> 31)


def kept_one(seed, drop_q16, i, step=0):
    """whether place i is kept, with Python's integers"""
    mask = (1 << 64) - 1
    key = fin(((((seed + step) & mask) ^ 0x3C6EF372FE94F82B) + 0x9E3779B97F4A7C15) & mask)
    word = fin((key + 0x9E3779B97F4A7C15 * (i // 4 + 1)) & mask)
    return (word >> 16 * (i % 4)) & 0xFFFF >= drop_q16


def kept(seed, drop_q16, first, n, step=0):
    """truth values of the places first .. first + n - 1"""
    with np.errstate(over="ignore"):
        mask = (1 << 64) - 1
        key = np.uint64(fin(((((seed + step) & mask) ^ 0x3C6EF372FE94F82B) + 0x9E3779B97F4A7C15) & mask))
        i = np.arange(first, first + n, dtype=np.uint64)
        z = key + np.uint64(0x9E3779B97F4A7C15) * (i // np.uint64(4) + np.uint64(1))
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        z = z ^ (z >> np.uint64(31))
        return (z >> (np.uint64(16) * (i % np.uint64(4)))) & np.uint64(0xFFFF) >= np.uint64(drop_q16)


def q16(p):
    return int(65536 * p + 0.5)


def factor(p):
    q = q16(p)
    return 0.0 if q == 65536 else 65536.0 / (65536 - q)


def in_memory_order(values, like):
    """a flat array of places in memory order as a tensor of the shape and strides of `like` (dense)"""
    out = torch.empty_strided(like.shape, like.stride(), dtype=torch.float64)
    torch.as_strided(out, (out.numel(),), (1,)).copy_(torch.from_numpy(np.ascontiguousarray(values)))
    return out


def mask_like(x, p, seed, step=0):
    """0 or the factor, in 64 bits, on the CPU"""
    return in_memory_order(kept(seed, q16(p), 0, x.numel(), step) * factor(p), x.cpu())


def depth(n):
    """additions in a row of fp32 sums over n channels of one position: those of a lane (at least 64 lanes share 512 values and more), of
    the lanes of a wave (6), and of the waves (16)"""
    return 32 + n / 64


def rms_forward(x, weight, residual, eps, axis, p=0.0, seed=0, step=0):
    """(y, h, rstd) and bounds of what they may differ by, in 64 bits on the CPU"""
    dt = x.dtype
    xs = x.cpu().double()
    if p:
        xs = xs * mask_like(x, p, seed, step)
    r = torch.zeros_like(xs) if residual is None else residual.cpu().double()
    h = xs + r
    n = x.shape[axis]
    w = torch.ones(n, dtype=torch.float64) if weight is None else weight.cpu().double()
    w = w.view(-1, *([1] * (x.dim() - 2))) if axis == 1 else w
    rstd = ((h * h).mean(axis, keepdim=True) + eps) ** -0.5
    y = h * rstd * w
    off_h = 2 * U * (xs.abs() + r.abs())                           # a product and an addition
    # half the relative error of the sum of squares (whose terms are off by twice what h is off), and of division, addition, root
    off_r = rstd * U * (depth(n) / 2 + 6) + rstd ** 3 * (off_h * h.abs()).mean(axis, keepdim=True)
    off_y = off_h * rstd * w.abs() + h.abs() * off_r * w.abs() + 4 * U * y.abs()
    sq = lambda t: t.squeeze(axis)
    return (y, h, sq(rstd)), (off_y * 1.01 + rounding(y, dt), off_h * 1.01 + rounding(h, dt), sq(off_r) * 1.01)


def rms_backward(dy, h, rstd, weight, dh, axis, p=0.0, seed=0, step=0, w_dtype=None):
    """(dx, dresidual, dweight) and bounds, from the h and rstd that the kernel is given"""
    dt = h.dtype
    d, x = dy.cpu().double(), h.cpu().double()
    r = rstd.cpu().double().unsqueeze(axis)
    n = h.shape[axis]
    w = torch.ones(n, dtype=torch.float64) if weight is None else weight.cpu().double()
    wb = w.view(-1, *([1] * (h.dim() - 2))) if axis == 1 else w
    g, xh = d * wb, x * r
    c, s = (g * xh).mean(axis, keepdim=True), (g * xh).abs().mean(axis, keepdim=True)
    e = torch.zeros_like(d) if dh is None else dh.cpu().double()
    dz = r * (g - xh * c) + e
    off = U * (6 * r * (g.abs() + (xh * c).abs()) + 2 * e.abs()) + r * xh.abs() * s * U * (depth(n) + 8)
    others = tuple(i for i in range(h.dim()) if i != axis % h.dim())
    dw, sw = (d * xh).sum(others), (d * xh).abs().sum(others)
    positions = h.numel() // n
    # additions in a row: a lane's share of the positions, then groups (128), workgroups (32) and rows of threads (16)
    off_w = U * (positions / 64 + 256) * sw
    wt = w_dtype or (dt if weight is None else weight.dtype)
    m = mask_like(h, p, seed, step) if p else torch.ones_like(dz)
    dx = dz * m
    return (dx, dz, dw), (off * m * 1.01 + 2 * U * dx.abs() + rounding(dx, dt), off * 1.01 + rounding(dz, dt), off_w * 1.01 + rounding(dw, wt))


def embedding_gradient(dy, idx, rows, scale, padding_idx=None, dtype=None):
    """dW and bounds in 64 bits on the CPU"""
    d = dy.cpu().double().reshape(-1, dy.shape[-1])
    t = idx.cpu().reshape(-1).long()
    there = (t >= 0) & (t < rows)
    if padding_idx is not None:
        there &= t != padding_idx
    dw = torch.zeros(rows, d.shape[1], dtype=torch.float64).index_add_(0, t[there], d[there])
    s = torch.zeros(rows, d.shape[1], dtype=torch.float64).index_add_(0, t[there], d[there].abs())
    n = torch.bincount(t[there], minlength=rows).double().unsqueeze(1)
    # additions in a row: 64 of a chunk, those of a wave over the chunks (at least 8 places each, 16 waves), 16 waves
    off = U * s * abs(scale) * (96 + n / 128) + 2 * U * (dw * scale).abs()
    return dw * scale, off * 1.01 + rounding(dw * scale, dtype or dy.dtype)


def close(got, want, bound):
    got = got.detach().cpu().double()
    assert got.shape == want.shape
    over = (got - want).abs() - bound
    assert torch.isfinite(got).all() and bool((over <= 0).all()), "off by %.3g where %.3g is allowed" % ((got - want).abs().flatten()[over.argmax()], bound.expand_as(over).flatten()[over.argmax()])
