"""Layer normalisation over channels (xconv_layernorm_fwd / _bwd, norm.py) against its formulas in 64 bits, at the sizes where
lanes, vectors, groups and workgroups end; refusals that need a device; a side stream; the module in a training step.

Tolerances come from the arithmetic: fp32 sums of chains of at most CHAIN additions (u = 2^-24 each, relative to the sum of the
absolute terms), a handful of roundings of every factor, and one rounding to the output's type."""
import numpy as np
import pytest
import torch

from paper_2106_06998_amd import binding as xb
from paper_2106_06998_amd import norm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TD = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24
UOUT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -25}
EPS = 1e-5


def chain(C):
    return 96 + C / 256          # a lane's own values in turn, then a tree over lanes and waves


def say(*a):
    print("[gpu-case]", *a, flush=True)


def draw(shape, seed, dtype, axis, offset=0.3):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    side = [1] * len(shape)
    side[axis] = shape[axis]
    x = x * (0.5 + torch.rand(side, generator=g)) + offset * torch.randn(side, generator=g) + offset
    dy = 0.1 * torch.randn(shape, generator=g)
    C = shape[axis]
    gamma, beta = 1 + 0.1 * torch.randn(C, generator=g), 0.1 * torch.randn(C, generator=g)
    return x.to(TD[dtype]), dy.to(TD[dtype]), gamma, beta


def along(t, ndim, axis):
    side = [1] * ndim
    side[axis] = -1
    return t.reshape(side)


def reference_fwd(x, gamma, beta, axis):
    """y, mean, rstd and the bounds of their errors, all in 64 bits."""
    x = x.double()
    C, nd = x.shape[axis], x.dim()
    mean = x.mean(axis, keepdim=True)
    var = ((x - mean) ** 2).mean(axis, keepdim=True)
    rstd = 1 / torch.sqrt(var + EPS)
    g = along(gamma.double(), nd, axis) if gamma is not None else torch.ones(1, dtype=torch.float64)
    b = along(beta.double(), nd, axis) if beta is not None else torch.zeros(1, dtype=torch.float64)
    xh = (x - mean) * rstd
    n = chain(C)
    dmean = n * U * x.abs().mean(axis, keepdim=True)
    drstd = rstd * (n * U + rstd * rstd * dmean * dmean)
    dxh = dmean * rstd + (8 * U + drstd / rstd) * xh.abs()
    return xh * g + b, mean, rstd, dxh * g.abs() + 8 * U * ((xh * g).abs() + b.abs()), dmean, drstd


def check_fwd(y, mean, rstd, x, gamma, beta, axis, dtype):
    wy, wm, wr, ty, tm, tr = reference_fwd(x, gamma, beta, axis)
    y, mean, rstd = y.cpu().double(), mean.cpu().double(), rstd.cpu().double()
    assert ((y - wy).abs() <= ty + (wy.abs() + ty) * UOUT[dtype] + TINY[dtype]).all(), float(((y - wy).abs() - ty - wy.abs() * UOUT[dtype]).max())
    assert ((mean - wm.squeeze(axis)).abs() <= (tm + U * wm.abs()).squeeze(axis)).all()
    assert ((rstd - wr.squeeze(axis)).abs() <= (tr + 4 * U * wr).squeeze(axis)).all()


def check_bwd(dx, dw, db, dy, x, mean, rstd, gamma, axis, dtype, wtype):
    nd, C = x.dim(), x.shape[axis]
    x, dy = x.double(), dy.double()
    mean, rstd = mean.cpu().double().unsqueeze(axis), rstd.cpu().double().unsqueeze(axis)
    g = dy * (along(gamma.double(), nd, axis) if gamma is not None else 1.0)
    xh = (x - mean) * rstd
    m1, m2 = g.mean(axis, keepdim=True), (g * xh).mean(axis, keepdim=True)
    want = rstd * (g - m1 - xh * m2)
    n = chain(C)
    tol = rstd * U * (8 * g.abs() + n * g.abs().mean(axis, keepdim=True) + xh.abs() * (n * (g * xh).abs().mean(axis, keepdim=True) + 8 * m2.abs()) + 8 * m1.abs())
    if dx is not None:
        assert ((dx.cpu().double() - want).abs() <= tol + (want.abs() + tol) * UOUT[dtype] + TINY[dtype]).all()
    others = [i for i in range(nd) if i != axis % nd]
    rows = x.numel() / C
    for got, term in ((dw, dy * xh), (db, dy)):
        if got is None:
            continue
        want, size = term.sum(others), term.abs().sum(others)
        t = (160 + rows / 1024) * U * size
        assert ((got.cpu().double() - want).abs() <= t + (want.abs() + t) * UOUT[wtype] + TINY[wtype]).all()


def run_case(shape, axis, dtype, wtype, seed, affine=True, offset=0.3, fmt=None):
    say("layer norm", shape, "axis", axis, dtype, wtype, "affine" if affine else "plain", fmt or "")
    x, dy, gamma, beta = draw(shape, seed, dtype, axis, offset)
    gamma, beta = (gamma.to(TD[wtype]), beta.to(TD[wtype])) if affine else (None, None)
    xd, dyd = x.to(DEV), dy.to(DEV)
    if fmt is not None:
        xd, dyd = xd.contiguous(memory_format=fmt), dyd.contiguous(memory_format=fmt)
    gd, bd = (gamma.to(DEV), beta.to(DEV)) if affine else (None, None)
    y, mean, rstd = norm.layer_norm_forward(xd, gd, bd, EPS, axis)
    dx, dw, db = norm.layer_norm_backward(dyd, xd, mean, rstd, gd, axis)
    torch.cuda.synchronize()
    assert y.dtype == TD[dtype] and dx.dtype == TD[dtype] and y.shape == x.shape and y.stride() == xd.stride() and dx.stride() == xd.stride()
    check_fwd(y, mean, rstd, x, gamma, beta, axis, dtype)
    check_bwd(dx, dw, db, dy, x, mean, rstd, gamma, axis, dtype, wtype if affine else dtype)
    # the same bits again: nothing depends on timing
    again = norm.layer_norm_backward(dyd, xd, mean, rstd, gd, axis)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), again))


# rows: below, at and past a vector, a group of lanes, a wave, a workgroup, the widest held row
@pytest.mark.parametrize("C", [1, 2, 3, 4, 5, 7, 8, 9, 16, 17, 31, 32, 33, 64, 65, 127, 128, 255, 256, 257, 500, 512, 513, 1000, 1023, 2047, 2048, 2049, 4097, 8191,
                               8200, 16384])
@pytest.mark.parametrize("dtype,wtype", [("f32", "f32"), ("bf16", "f32"), ("f16", "f16")])
def test_rows_of_every_length(C, dtype, wtype):
    run_case((11, C), -1, dtype, wtype, 100 + C)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_longer_than_the_registers(dtype):
    run_case((5, 40001), -1, dtype, "f32", 7)
    run_case((1100, 33001), -1, dtype, "f32", 8)          # more rows than workgroups that leave partial sums


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 63, 64, 65, 1000, 5003, 70001])
def test_any_number_of_rows(rows):
    run_case((rows, 24), -1, "f32", "f32", 200 + rows)
    run_case((rows, 40), -1, "f16", "f32", 300 + rows)


@pytest.mark.parametrize("B,C,H,W", [(1, 1, 1, 2), (2, 3, 1, 5), (3, 5, 7, 7), (1, 16, 4, 4), (7, 37, 19, 23), (2, 64, 32, 32), (5, 100, 3, 3), (2, 129, 28, 28),
                                     (2, 256, 28, 28), (3, 511, 5, 9), (2, 520, 8, 8), (1, 1000, 6, 7), (1, 1030, 4, 9), (1, 2500, 5, 5), (300, 20, 2, 1)])
@pytest.mark.parametrize("dtype,wtype", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32")])
def test_planes(B, C, H, W, dtype, wtype):
    run_case((B, C, H, W), 1, dtype, wtype, B + C + H)


def test_many_planes_per_workgroup():
    run_case((64, 24, 40, 40), 1, "bf16", "f32", 5)
    run_case((40, 700, 13, 31), 1, "f16", "f32", 6)


def test_channels_last_volumes_and_two_axes():
    run_case((3, 20, 6, 5), 1, "f16", "f32", 1, fmt=torch.channels_last)
    run_case((2, 20, 3, 6, 5), 1, "f32", "f32", 2, fmt=torch.channels_last_3d)
    run_case((2, 20, 3, 6, 5), 1, "bf16", "f32", 3)
    run_case((6, 20), 1, "f32", "f32", 4)
    run_case((4, 5, 20), -1, "f32", "f32", 5)
    run_case((4, 20, 5), 1, "f32", "f32", 6)


def test_without_parameters_and_far_from_zero():
    run_case((9, 77), -1, "f32", "f32", 1, affine=False)
    run_case((2, 21, 5, 7), 1, "bf16", "bf16", 2, affine=False)
    run_case((9, 300), -1, "f32", "f32", 3, offset=1000.0)
    run_case((2, 48, 6, 6), 1, "f32", "f32", 4, offset=1000.0)


def test_subsets_of_the_gradients():
    x, dy, gamma, _ = draw((33, 50), 3, "f32", -1)
    xd, dyd, gd = x.to(DEV), dy.to(DEV), gamma.to(DEV)
    _, mean, rstd = norm.layer_norm_forward(xd, gd, None, EPS)
    full = norm.layer_norm_backward(dyd, xd, mean, rstd, gd)
    for need in ((True, False, False), (False, True, False), (False, False, True), (True, True, False), (False, False, False)):
        got = norm.layer_norm_backward(dyd, xd, mean, rstd, gd, need=need)
        for n, a, b in zip(need, got, full):
            assert (a is None) if not n else torch.equal(a, b)
    xp = x[:32].reshape(2, 16, 50).transpose(1, 2).contiguous().to(DEV)      # [2, 50, 16] planes
    dp = dy[:32].reshape(2, 16, 50).transpose(1, 2).contiguous().to(DEV)
    _, mean, rstd = norm.layer_norm_forward(xp, gd, None, EPS, 1)
    full = norm.layer_norm_backward(dp, xp, mean, rstd, gd, 1)
    for need in ((True, False, False), (False, True, False), (False, False, True)):
        got = norm.layer_norm_backward(dp, xp, mean, rstd, gd, 1, need)
        for n, a, b in zip(need, got, full):
            assert (a is None) if not n else torch.equal(a, b)


def test_equal_values_and_non_finite_positions_stay_where_they_are():
    for shape, axis in (((6, 40), -1), ((2, 40, 3, 7), 1)):
        x, dy, gamma, beta = draw(shape, 5, "f32", axis)
        if axis == 1:
            x[0, :, 1, 2] = 3.0
            x[1, 4, 0, 1] = float("inf")
            x[1, 7, 2, 6] = float("nan")
        else:
            x[1] = 3.0
            x[3, 4] = float("inf")
            x[5, 7] = float("nan")
        xd, dyd, gd, bd = (t.to(DEV) for t in (x, dy, gamma, beta))
        y, mean, rstd = norm.layer_norm_forward(xd, gd, bd, EPS, axis)
        dx, _, db = norm.layer_norm_backward(dyd, xd, mean, rstd, gd, axis)
        torch.cuda.synchronize()
        fine = torch.isfinite(x).all(axis)
        for t in (y, dx):
            t = t.cpu()
            assert torch.equal(torch.isfinite(t).all(axis), fine)
        y = y.cpu()
        same = y[0, :, 1, 2] if axis == 1 else y[1]
        assert torch.equal(same, beta)
        assert torch.isfinite(db).all()


def test_views_and_other_orders():
    x, dy, gamma, beta = draw((64, 97), 9, "f16", -1)
    gd, bd = gamma.to(DEV), beta.to(DEV)
    big = torch.zeros(64, 200, dtype=torch.float16, device=DEV)
    big[:, 51:148] = x.to(DEV)
    view, dyt = big[:, 51:148], dy.t().contiguous().to(DEV).t()
    y, mean, rstd = norm.layer_norm_forward(view, gd, bd, EPS)
    dx, dw, db = norm.layer_norm_backward(dyt, view, mean, rstd, gd)
    torch.cuda.synchronize()
    check_fwd(y, mean, rstd, x, gamma, beta, -1, "f16")
    check_bwd(dx, dw, db, dy, x, mean, rstd, gamma, -1, "f16", "f32")
    # a storage offset that is no multiple of 16 bytes, and strided parameters
    flat = torch.zeros(64 * 97 + 3, dtype=torch.float16, device=DEV)
    flat[3:] = x.reshape(-1).to(DEV)
    g2 = torch.zeros(97, 2, device=DEV)
    g2[:, 1] = gd
    y2, _, _ = norm.layer_norm_forward(flat[3:].view(64, 97), g2[:, 1], bd, EPS)
    assert torch.equal(y, y2)


def test_nothing_and_one_position():
    for shape, axis in (((0, 12), -1), ((0, 12, 3, 3), 1), ((2, 12, 0, 3), 1)):
        x = torch.empty(shape, device=DEV)
        y, mean, rstd = norm.layer_norm_forward(x, None, None, EPS, axis)
        dx, dw, db = norm.layer_norm_backward(y, x, mean, rstd, None, axis)
        assert y.shape == x.shape and mean.numel() == 0 and dx.shape == x.shape
        assert torch.equal(dw.cpu(), torch.zeros(12)) and torch.equal(db.cpu(), torch.zeros(12))
    run_case((1, 12), -1, "f32", "f32", 4)
    run_case((1, 12, 1, 1), 1, "bf16", "f32", 4)


def test_in_place_and_guard_values():
    for outer, C, inner in ((37, 53, 1), (3, 53, 11), (2, 1100, 9), (3, 40000, 1)):
        x, dy, gamma, beta = draw((outer, C, inner), 12, "f32", 1)
        n = x.numel()
        buf = torch.full((n + 8,), 7.0, device=DEV)
        buf[4:4 + n] = x.reshape(-1).to(DEV)
        d = xb.make_norm_desc(outer, C, inner, "f32", "f32", EPS)
        gd, bd = gamma.to(DEV), beta.to(DEV)
        out = torch.full((n,), float("nan"), device=DEV)
        stats = torch.empty(2, outer * inner, device=DEV)
        xb.xconv_layernorm_fwd(d, buf[4:4 + n], gd, bd, out, stats[0], stats[1])
        xb.xconv_layernorm_fwd(d, buf[4:4 + n], gd, bd, buf[4:4 + n])
        torch.cuda.synchronize()
        assert torch.equal(buf[4:4 + n], out) and (buf[:4] == 7).all() and (buf[-4:] == 7).all()
        ws = xb.alloc_bytes(xb.xconv_layernorm_workspace_bytes(d))
        xd, dyd = x.reshape(-1).to(DEV), dy.reshape(-1).to(DEV)
        pair = torch.full((2, C), float("nan"), device=DEV)
        xb.xconv_layernorm_bwd(d, dyd, xd, stats[0], stats[1], gd, out, pair[0], pair[1], ws)
        xb.xconv_layernorm_bwd(d, dyd, xd, stats[0], stats[1], gd, dyd, None, None, None)
        torch.cuda.synchronize()
        assert torch.equal(dyd, out) and torch.isfinite(pair).all()


def test_past_32_bit_offsets():
    """2^31 + elements: the last rows lie past a 32-bit element offset."""
    C, rows = 8192, (1 << 18) + 3
    say("layer norm of", rows, "rows of", C, "f16")
    x = torch.zeros(rows, C, dtype=torch.float16, device=DEV)
    tail, dy, gamma, beta = draw((5, C), 21, "f16", -1)
    x[-5:] = tail.to(DEV)
    gd, bd = gamma.to(DEV), beta.to(DEV)
    y, mean, rstd = norm.layer_norm_forward(x, gd, bd, EPS)
    torch.cuda.synchronize()
    check_fwd(y[-5:], mean[-5:], rstd[-5:], tail, gamma, beta, -1, "f16")
    del y
    g = torch.zeros_like(x)
    g[-5:] = dy.to(DEV)
    dx, dw, db = norm.layer_norm_backward(g, x, mean, rstd, gd)
    torch.cuda.synchronize()
    check_bwd(dx[-5:], dw, db, dy, tail, mean[-5:], rstd[-5:], gamma, -1, "f16", "f32")
    assert not dx[:1000].any()


def test_gradient_against_differences():
    """The directional derivative of sum(c * y) along v from the forward pass itself: (f(t) - f(-t)) / 2t has an error of t^2 f'''/6
    (values of order one: below 1e-3 of it at t = 1e-2) and of the rounding of y over t (2^-24 / 1e-2 a term, below 1e-4 of the sum)."""
    for shape, axis in (((40, 30), -1), ((2, 30, 4, 5), 1)):
        x, c, gamma, beta = (t.to(DEV) for t in draw(shape, 31, "f32", axis))
        v, _, vg, vb = (t.to(DEV) for t in draw(shape, 32, "f32", axis))
        c = c * 10
        xp, gp, bp = (t.clone().requires_grad_() for t in (x, gamma, beta))
        (norm.layer_norm(xp, gp, bp, EPS, axis) * c).sum().backward()
        f = lambda t: float((norm.layer_norm_forward(x + t * v, gamma + t * vg, beta + t * vb, EPS, axis)[0].double() * c.double()).sum())
        t = 1e-2
        want = (f(t) - f(-t)) / (2 * t)
        got = float((xp.grad.double() * v).sum() + (gp.grad.double() * vg).sum() + (bp.grad.double() * vb).sum())
        size = float((xp.grad.double() * v).abs().sum() + (gp.grad.double() * vg).abs().sum() + (bp.grad.double() * vb).abs().sum())
        assert abs(got - want) <= 2e-3 * size, (got, want, size)


def test_on_a_side_stream_and_in_a_graph():
    x, dy, gamma, beta = (t.to(DEV) for t in draw((6, 33, 9, 11), 41, "f16", 1))
    want = norm.layer_norm_forward(x, gamma, beta, EPS, 1)
    want += norm.layer_norm_backward(dy, x, want[1], want[2], gamma, 1)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = norm.layer_norm_forward(x, gamma, beta, EPS, 1)
        got += norm.layer_norm_backward(dy, x, got[1], got[2], gamma, 1)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = norm.layer_norm_forward(x, gamma, beta, EPS, 1)
        out += norm.layer_norm_backward(dy, x, out[1], out[2], gamma, 1)
    keep = x.clone()
    for k in range(3):
        x.copy_(keep * (1 + k))
        graph.replay()
        torch.cuda.synchronize()
        eager = norm.layer_norm_forward(x, gamma, beta, EPS, 1)
        eager += norm.layer_norm_backward(dy, x, eager[1], eager[2], gamma, 1)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager))


def test_module_matches_the_function_and_its_types():
    x, dy, gamma, beta = draw((3, 24, 5, 6), 51, "f16", 1)
    m = norm.XLayerNorm(24, axis=1, device=DEV)
    with torch.no_grad():
        m.weight.copy_(gamma)
        m.bias.copy_(beta)
    xd = x.to(DEV).requires_grad_()
    y = m(xd)
    y.backward(dy.to(DEV))
    torch.cuda.synchronize()
    check_fwd(y.detach(), *norm.layer_norm_forward(xd.detach(), m.weight.detach(), m.bias.detach(), EPS, 1)[1:], x, gamma, beta, 1, "f16")
    assert xd.grad.dtype == torch.float16 and m.weight.grad.dtype == torch.float32 and m.bias.grad.dtype == torch.float32
    assert np.isfinite(m.weight.grad.cpu().numpy()).all()
    plain = norm.XLayerNorm(24, axis=-1, elementwise_affine=False)
    assert plain.weight is None and plain(x.to(DEV).permute(0, 2, 3, 1)).shape == (3, 5, 6, 24)


def test_refusals_on_the_device():
    x = torch.zeros(4, 8, device=DEV)
    with pytest.raises(RuntimeError, match="not supported"):
        norm.layer_norm(x.double())
    with pytest.raises(RuntimeError, match="channels are the last axis"):
        norm.layer_norm_forward(torch.zeros(2, 3, 4, 5, device=DEV), axis=2)
    with pytest.raises(RuntimeError, match="parameters of 8 channels"):
        norm.layer_norm_forward(x, torch.ones(7, device=DEV))
    with pytest.raises(RuntimeError, match="float32 or of the input's type"):
        norm.layer_norm_forward(x, torch.ones(8, device=DEV, dtype=torch.float16))
    with pytest.raises(RuntimeError, match="of one type"):
        h = x.half()
        norm.layer_norm_forward(h, torch.ones(8, device=DEV), torch.ones(8, device=DEV, dtype=torch.float16))
    with pytest.raises(RuntimeError, match="on the input's device"):
        norm.layer_norm_forward(x, torch.ones(8))
    with pytest.raises(xb.XConvError):
        norm.layer_norm_forward(x, eps=-1.0)
    y, mean, rstd = norm.layer_norm_forward(x)
    with pytest.raises(RuntimeError, match="another shape"):
        norm.layer_norm_backward(torch.zeros(4, 9, device=DEV), x, mean, rstd)
    with pytest.raises(RuntimeError, match="forward pass"):
        norm.layer_norm_backward(x, x, mean[:3], rstd)
    with pytest.raises(RuntimeError, match="8 channels"):
        norm.XLayerNorm(8)(torch.zeros(2, 9, device=DEV))


@pytest.mark.parametrize("shape,axis", [((6, 37), -1), ((9, 500), -1), ((5, 1300), -1), ((2, 37, 5, 5), 1), ((1, 1100, 3, 4), 1)])
def test_backward_where_mean_times_rstd_leaves_the_range(shape, axis):
    """Positions with one value of 2^122 in all channels and an rstd of 10^5: x - mean and what follows from it is 0, everything
    is finite.  Lanes that have no channel see that mean as well."""
    say("layer norm", shape, "constant positions")
    x = torch.full(shape, 2.0 ** 122)
    dy = draw(shape, 4, "f32", axis)[1]
    stat = [s for i, s in enumerate(shape) if i != axis % len(shape)]
    mean, rstd = torch.full(stat, 2.0 ** 122), torch.full(stat, 1e5)
    dx, dw, db = norm.layer_norm_backward(dy.to(DEV), x.to(DEV), mean.to(DEV), rstd.to(DEV), None, axis)
    torch.cuda.synchronize()
    assert not dw.any()
    size = dy.double()
    want = 1e5 * (size - size.mean(axis, keepdim=True))
    tol = 1e5 * U * (8 * size.abs() + chain(shape[axis]) * size.abs().mean(axis, keepdim=True)) + 4 * U * want.abs()
    assert ((dx.cpu().double() - want).abs() <= tol).all()
