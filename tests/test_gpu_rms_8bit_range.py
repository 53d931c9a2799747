"""The 8-bit root-mean-square norm where its factors are far apart: positions of zeros and of tiny values under a tiny eps (rstd is large, and
so is what the scale's least magnitude divides), and its bits from call to call."""
import pytest
import torch

import token_reference as ref
from paper_2106_06998_amd import norm as N

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TOP = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}
LEAST = 2.0 ** -100
# groups of 4 to 1024 lanes with one to eight vectors, rows that are read again; planes of 4 to 16 waves and those that are read again
SHAPES = [((5, 3), -1), ((6, 40), -1), ((6, 300), -1), ((5, 1000), -1), ((5, 2500), -1), ((5, 5001), -1), ((5, 12000), -1), ((5, 40003), -1),
          ((3, 3, 1, 2), 1), ((3, 20, 5, 7), 1), ((2, 130, 4, 6), 1), ((2, 300, 4, 6), 1), ((2, 700, 3, 5), 1), ((2, 1100, 3, 5), 1)]


def _normal(shape, dtype, seed, scale=1.0):
    return (scale * torch.randn(shape, generator=torch.Generator().manual_seed(seed))).to(dtype).to(DEV)


def _ids(v):
    return "x".join(map(str, v)) if isinstance(v, tuple) else None


@pytest.mark.parametrize("out", sorted(TOP, key=str))
@pytest.mark.parametrize("eps", [1e-12, 1e-14, 1e-20])
@pytest.mark.parametrize("shape,axis", SHAPES, ids=_ids)
def test_positions_of_zeros(shape, axis, eps, out):
    """Y is zero there, so Q = Y / scale is, and the scale is the least one; the others are what they are without them"""
    for dtype in sorted(TYPES):
        x = _normal(shape, TYPES[dtype], 1)
        clean = N.rms_norm_8bit(x, None, None, eps, axis, out)
        pos = (1,) if axis == -1 else (1, slice(None), 0, 1)
        z = x.clone()
        z[pos] = 0
        for residual in (None, torch.zeros_like(z)):
            q, scale, _ = N.rms_norm_8bit(z, None, residual, eps, axis, out)
            spos = (1,) if axis == -1 else (1, 0, 1)
            assert bool((q[pos].float() == 0).all()), dtype
            assert float(scale[spos]) == float(torch.tensor(LEAST) / TOP[out])
            other, sother = torch.ones(shape, dtype=torch.bool, device=DEV), torch.ones(scale.shape, dtype=torch.bool, device=DEV)
            other[pos], sother[spos] = False, False
            assert torch.equal(q.float()[other], clean[0].float()[other]) and torch.equal(scale[sother], clean[1][sother])


@pytest.mark.parametrize("out", sorted(TOP, key=str))
@pytest.mark.parametrize("gain", [1e-28, 1e-30, 1e-32])
@pytest.mark.parametrize("shape,axis", SHAPES, ids=_ids)
def test_tiny_rows_and_gains(shape, axis, gain, out):
    """rstd some 1e7, Y at the least magnitude of a scale and on both sides of it; an h gamma below 2^-126 is off by half its least step,
    2^-150, which rstd multiplies"""
    for dtype, eps in (("f32", 1e-14), ("bf16", 1e-14), ("f32", 1e-16)):
        x = _normal(shape, TYPES[dtype], 1, 1e-7)
        w = gain * (1 + 0.3 * _normal((shape[axis],), torch.float32, 3))
        q, scale, _ = N.rms_norm_8bit(x, w, None, eps, axis, out)
        (y, _, rstd), _ = ref.rms_forward(x, w, None, eps, axis)
        _, (off, _, _) = ref.rms_forward(x.float(), w, None, eps, axis)
        off = off + 2.0 ** -150 * rstd.unsqueeze(axis) * 1.01
        s, top = scale.cpu().double().unsqueeze(axis), TOP[out]
        most = y.abs().amax(axis, keepdim=True).clamp(min=LEAST)
        assert bool(((s * top - most).abs() <= off.amax(axis, keepdim=True) + 4 * ref.U * most).all())
        # half a step (e4m3: 2^-4 of the value, below 2^-6 2^-10; int8: 1/2) and the roundings of the factors and of two products
        v = q.cpu().float().double()
        assert bool(torch.isfinite(v).all())
        step = (v.abs() * 2.0 ** -3).clamp(min=2.0 ** -9) / 2 if out == torch.float8_e4m3fn else torch.full_like(v, 0.5)
        assert bool(((v * s - y).abs() <= step * s * 1.001 + off + 6 * ref.U * y.abs()).all())


@pytest.mark.parametrize("out", sorted(TOP, key=str))
@pytest.mark.parametrize("shape,axis", [((2000, 5001), -1), ((3000, 300), -1), ((40, 64, 13, 11), 1)], ids=_ids)
def test_the_same_bits_every_time(shape, axis, out):
    x, r, w = _normal(shape, torch.float16, 1), _normal(shape, torch.float16, 2), 1 + 0.3 * _normal((shape[axis],), torch.float32, 3)
    for residual in (None, r):
        first = N.rms_norm_8bit(x, w, residual, 1e-6, axis, out)
        for _ in range(8):
            again = N.rms_norm_8bit(x, w, residual, 1e-6, axis, out)
            assert torch.equal(again[0].view(torch.uint8), first[0].view(torch.uint8)) and all(torch.equal(a, b) for a, b in zip(again[1:], first[1:]))
