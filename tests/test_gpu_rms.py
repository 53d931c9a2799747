"""Root-mean-square norm with residual and dropout against its definition in 64 bits; bounds are those of fp32 arithmetic and one
rounding (token_reference.py)."""
import pytest
import torch

import token_reference as ref
from paper_2106_06998_amd import binding as xb
from paper_2106_06998_amd import norm as N
from paper_2106_06998_amd.dropout import dropout_forward

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6


def _normal(shape, dtype, seed, scale=1.0):
    return (scale * torch.randn(shape, generator=torch.Generator().manual_seed(seed))).to(dtype).to(DEV)


# every group of lanes, vectors a lane, and the rows that are read again; whole and ragged lengths
ROWS = [(1, 1), (3, 2), (5, 3), (7, 7), (9, 8), (130, 32), (131, 33), (64, 64), (33, 100), (50, 127), (17, 256), (19, 300), (9, 512), (5, 1000), (6, 1024), (3, 2001), (4, 2048),
        (3, 4096), (2, 5001), (3, 8191), (2, 8192), (2, 12000), (1, 16385), (2, 20000), (1, 33000), (2, 40003), (700, 48), (1500, 20),
        (3, 1500), (3, 2500), (2, 3000), (2, 6001), (2, 10000), (2, 14002), (1, 24000), (1, 32000)]
PLANES = [(1, 1, 1, 2), (2, 3, 1, 3), (2, 5, 2, 2), (3, 8, 4, 4), (2, 17, 5, 7), (1, 32, 3, 3), (2, 33, 8, 8), (2, 64, 6, 5), (1, 100, 7, 9), (2, 128, 4, 4), (1, 200, 5, 5), (1, 256, 7, 7),
          (1, 300, 3, 11), (1, 512, 4, 5), (1, 700, 3, 5), (1, 1024, 5, 5), (1, 1500, 3, 7), (40, 16, 12, 10)]


def _case(shape, axis, dtype, wdtype, residual, p, eps=EPS):
    dt, wt = TYPES[dtype], TYPES[wdtype]
    n = shape[axis]
    x = _normal(shape, dt, 1) + _normal((n,) if axis == -1 else (1, n) + (1,) * (len(shape) - 2), dt, 2)
    w = (1 + 0.3 * _normal((n,), torch.float32, 3)).to(wt)
    r = _normal(shape, dt, 4) if residual else None
    seed = 1000 + n
    y, h, rstd = N.rms_norm_forward(x, w, r, eps, axis, p, seed)
    want, off = ref.rms_forward(x, w, r, eps, axis, p, seed)
    ref.close(y, want[0], off[0])
    if residual or p:
        ref.close(h, want[1], off[1])
    else:
        assert h is x
    ref.close(rstd, want[2], off[2])
    dy, dh = _normal(shape, dt, 5, 0.1), _normal(shape, dt, 6, 0.1) if residual else None
    dx, dr, dw = N.rms_norm_backward(dy, h, rstd, w, dh, axis, p, seed)
    assert p > 0 or dx is dr
    want, off = ref.rms_backward(dy, h, rstd, w, dh, axis, p, seed)
    for g, a, b in zip((dx, dr, dw), want, off):
        ref.close(g, a, b)
    # what is not asked for changes nothing of the rest
    for need in ((True, False, False), (False, True, True), (False, False, True)):
        some = N.rms_norm_backward(dy, h, rstd, w, dh, axis, p, seed, need=need)
        for g, a, wanted in zip(some, (dx, dr, dw), need):
            assert (g is None) == (not wanted) and (g is None or torch.equal(g, a))
    # dropping from the stored dresidual rounds once more than dx
    if p:
        again = dropout_forward(dr, p, seed)
        assert bool(((again == 0) | (dx != 0) | (again.abs() < 1e-3)).all())


@pytest.mark.parametrize("dtype,wdtype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("shape", ROWS, ids=lambda s: "%dx%d" % s)
def test_rows(shape, dtype, wdtype):
    _case(shape, -1, dtype, wdtype, True, 0.2)
    if dtype == wdtype:
        _case(shape, -1, dtype, wdtype, False, 0.0)


@pytest.mark.parametrize("dtype,wdtype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("shape", PLANES, ids=lambda s: "x".join(map(str, s)))
def test_planes(shape, dtype, wdtype):
    _case(shape, 1, dtype, wdtype, True, 0.2)
    if dtype == wdtype:
        _case(shape, 1, dtype, wdtype, False, 0.0)


@pytest.mark.parametrize("residual,p", [(True, 0.0), (False, 0.3), (False, 1.0)])
def test_residual_or_dropout_alone(residual, p):
    _case((37, 200), -1, "bf16", "f32", residual, p)
    _case((3, 40, 5, 6), 1, "f16", "f32", residual, p)


def test_layouts_and_copies():
    """channels-last tensors, volumes, gaps, offsets: results as of dense copies, in the input's layout"""
    x, r = _normal((3, 24, 5, 4), torch.bfloat16, 1), _normal((3, 24, 5, 4), torch.bfloat16, 2)
    w = _normal((24,), torch.float32, 3)
    xl = x.contiguous(memory_format=torch.channels_last)
    y, h, rstd = N.rms_norm_forward(xl, w, r, EPS, 1, 0.25, 9)
    assert y.is_contiguous(memory_format=torch.channels_last) and h.is_contiguous(memory_format=torch.channels_last) and rstd.shape == (3, 5, 4)
    want, off = ref.rms_forward(xl, w, r, EPS, 1, 0.25, 9)
    for g, a, b in zip((y, h, rstd), want, off):
        ref.close(g, a, b)
    rows = xl.permute(0, 2, 3, 1)
    same = N.rms_norm_forward(rows, w, r.permute(0, 2, 3, 1), EPS, -1, 0.25, 9)
    assert torch.equal(same[0], y.permute(0, 2, 3, 1))
    dy = _normal((3, 24, 5, 4), torch.bfloat16, 4)
    got = N.rms_norm_backward(dy, h, rstd, w, None, 1, 0.25, 9)
    want, off = ref.rms_backward(dy, h, rstd, w, None, 1, 0.25, 9)
    for g, a, b in zip(got, want, off):
        ref.close(g, a, b)
    v = _normal((2, 8, 3, 4, 5), torch.float32, 5)
    a = N.rms_norm_forward(v, None, None, EPS, 1)[0]
    b = N.rms_norm_forward(v.contiguous(memory_format=torch.channels_last_3d), None, None, EPS, 1)[0]
    want, off = ref.rms_forward(v, None, None, EPS, 1)
    ref.close(a, want[0], off[0])
    ref.close(b, want[0], off[0])
    g = _normal((10, 50), torch.float32, 6)
    for t in (g[:, 3:40], g.t(), g[::2], g[1:, 1:].t(), _normal((1, 30), torch.float32, 7).expand(4, 30)):
        assert torch.equal(N.rms_norm_forward(t)[0], N.rms_norm_forward(t.contiguous())[0])
    flat = _normal((5 * 33 + 1,), torch.float16, 8)
    off1 = flat[1:].view(5, 33)                             # not aligned to 4 bytes
    assert torch.equal(N.rms_norm_forward(off1)[0], N.rms_norm_forward(off1.clone())[0])


@pytest.mark.parametrize("axis,shape", [(-1, (6, 40)), (1, (2, 40, 3, 3))])
def test_what_is_not_finite(axis, shape):
    x = _normal(shape, torch.float32, 1)
    at = (2, 7) if axis == -1 else (1, 7, 1, 2)
    pos = 2 if axis == -1 else (1, slice(None), 1, 2)
    clean = N.rms_norm_forward(x, None, None, EPS, axis)[0]
    for bad in (float("nan"), float("inf"), -float("inf")):
        z = x.clone()
        z[at] = bad
        y, _, rstd = N.rms_norm_forward(z, None, None, EPS, axis)
        q, scale, _ = N.rms_norm_8bit(z, None, None, EPS, axis)
        i8 = N.rms_norm_8bit(z, None, None, EPS, axis, torch.int8)
        assert bool(torch.isnan(y[at])) and bool(torch.isnan((q.float() * scale.unsqueeze(axis))[pos]).all())
        assert bool(torch.isnan(i8[1]).any()) and int(torch.isnan(scale).sum()) == int(torch.isnan(i8[1]).sum()) == 1
        other = torch.ones(shape, dtype=torch.bool, device=DEV)
        other[pos] = False
        assert torch.equal(y[other], clean[other])
    # rows of zeros: y is zero with eps, the gradient finite
    z = x.clone()
    z[pos] = 0
    y, h, rstd = N.rms_norm_forward(z, None, None, EPS, axis)
    assert bool((y[pos] == 0).all())
    dx, _, _ = N.rms_norm_backward(torch.ones_like(y), h, rstd, None, None, axis)
    assert bool(torch.isfinite(dx).all())
    q, scale, _ = N.rms_norm_8bit(z, None, None, EPS, axis)
    assert bool((q.float()[pos] == 0).all()) and bool((scale > 0).all())


def test_empty():
    for shape, axis in (((0, 16), -1), ((0, 16, 2, 2), 1), ((3, 16, 0, 2), 1)):
        x, w = torch.empty(shape, device=DEV), torch.ones(16, device=DEV)
        y, h, rstd = N.rms_norm_forward(x, w, x, EPS, axis, 0.1, 1)
        assert y.shape == h.shape == x.shape and rstd.numel() == 0
        dx, dr, dw = N.rms_norm_backward(y, h, rstd, w, h, axis, 0.1, 1)
        assert dx.shape == x.shape and bool((dw == 0).all())
        q, scale, _ = N.rms_norm_8bit(x, w, None, EPS, axis)
        assert q.shape == x.shape and scale.numel() == 0


@pytest.mark.parametrize("out", [torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("shape,axis", [((1, 1), -1), ((3, 5), -1), ((5, 64), -1), ((9, 300), -1), ((1, 4096), -1), ((4, 5001), -1), ((2, 9000), -1), ((2, 40001), -1),
                                        ((2, 1500), -1), ((2, 2500), -1), ((2, 2999), -1), ((2, 6000), -1), ((2, 12000), -1), ((2, 17000), -1), ((2, 21000), -1), ((2, 32000), -1),
                                        ((2, 3, 1, 2), 1), ((2, 20, 5, 7), 1), ((1, 130, 4, 6), 1), ((1, 700, 3, 5), 1), ((1, 1100, 2, 5), 1)])
def test_8_bits(shape, axis, dtype, out):
    dt = TYPES[dtype]
    x, r = _normal(shape, dt, 1), _normal(shape, dt, 2)
    w = (1 + 0.3 * _normal((shape[axis],), torch.float32, 3))
    for res in (None, r):
        q, scale, h = N.rms_norm_8bit(x, w, res, EPS, axis, out)
        assert q.dtype == out and scale.dtype == torch.float32 and (h is x) == (res is None)
        (y, hw, _), (_, off_h, _) = ref.rms_forward(x, w, res, EPS, axis)
        _, (off32, _, _) = ref.rms_forward(x.float(), w, None if res is None else res.float(), EPS, axis)
        if res is not None:
            ref.close(h, hw, off_h)
        s = scale.cpu().double().unsqueeze(axis)
        top = 448 if out == torch.float8_e4m3fn else 127
        most = y.abs().amax(axis, keepdim=True)
        off_s = off32.amax(axis, keepdim=True) + 4 * ref.U * most
        assert bool(((s * top - most).abs() <= off_s).all())
        # half a step: of e4m3 2^-4 of the value, below 2^-6 2^-10; of int8 1/2; the quotient is off by two roundings more
        v = q.cpu().float().double()
        step = (v.abs() * 2.0 ** -3).clamp(min=2.0 ** -9) / 2 if out == torch.float8_e4m3fn else torch.full_like(v, 0.5)
        assert bool(((v * s - y).abs() <= step * s * 1.001 + off32 + 4 * ref.U * y.abs()).all())
        assert bool((v.abs().amax(axis) == top).all())


def test_8_bits_round_as_torch():
    """q is what torch makes of the same quotient, ties to even among them: with every y and scale a short number nothing else rounds"""
    n = 256
    y = torch.zeros(n)
    y[0], y[1] = 448.0, 1.0
    y[2:] = torch.arange(n - 2) * 0.25 - 30
    # one row whose norm is 1 up to a power of two: weights carry the values
    x = torch.ones(1, n, device=DEV)
    q, scale, _ = N.rms_norm_8bit(x, y.to(DEV), None, 0.0)
    assert float(scale) == 1.0 and torch.equal(q.float().cpu()[0], y.to(torch.float8_e4m3fn).float())
    y = torch.cat([torch.tensor([127.0, -126.5]), torch.arange(254) * 0.5 - 63.25])
    q, scale, _ = N.rms_norm_8bit(x, y.to(DEV), None, 0.0, dtype=torch.int8)
    assert float(scale) == 1.0 and torch.equal(q.float().cpu()[0], torch.round(y))


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("p", [0.0, 0.25])
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_autograd(dtype, p, residual):
    dt = TYPES[dtype]
    x, r = _normal((4, 48, 3, 5), dt, 1).requires_grad_(), _normal((4, 48, 3, 5), dt, 2).requires_grad_() if residual else None
    w = (1 + 0.3 * _normal((48,), torch.float32, 3)).requires_grad_()
    a, b = _normal((4, 48, 3, 5), dt, 4), _normal((4, 48, 3, 5), dt, 5)
    out = N.rms_norm(x, w, r, EPS, 1, p, 7)
    y, h = out if residual else (out, None)
    _, hs, rstd = N.rms_norm_forward(x.detach(), w.detach(), None if r is None else r.detach(), EPS, 1, p, 7)
    torch.autograd.backward([y, h], [a, b]) if residual else y.backward(a)
    want = N.rms_norm_backward(a, hs, rstd, w.detach(), b if residual else None, 1, p, 7)
    for g, v in zip((x.grad, r.grad if residual else None, w.grad), want):
        assert g is None or torch.equal(g, v)
    assert not residual or x.grad.data_ptr() != r.grad.data_ptr()         # (one tensor came back for both without dropout)
    if residual:
        # h alone, y alone, with broadcast gradients and of another type
        for outputs in ("h", "y"):
            x.grad = r.grad = w.grad = None
            y, h = N.rms_norm(x, w, r, EPS, 1, p, 7)
            (h if outputs == "h" else y).sum().backward()
            one = torch.ones_like(hs)
            want = N.rms_norm_backward(one if outputs == "y" else torch.zeros_like(one), hs, rstd, w.detach(), one if outputs == "h" else None, 1, p, 7)
            assert torch.equal(x.grad, want[0]) and torch.equal(r.grad, want[1]) and torch.equal(w.grad, want[2])
    # the same tensor as branch and residual
    z = x.detach().clone().requires_grad_()
    y, h = N.rms_norm(z, None, z, EPS, 1)
    (y.float().sum() + h.float().sum()).backward()
    _, hs, rstd = N.rms_norm_forward(z.detach(), None, z.detach(), EPS, 1)
    dz = N.rms_norm_backward(torch.ones_like(z), hs, rstd, None, torch.ones_like(z), 1)[0]
    assert torch.equal(z.grad, (dz + dz))


def test_gradient_against_differences():
    """along random directions, of the definition in 64 bits: central differences are off by 1e-12 (step 1e-6) and 1e-10 (rounding)"""
    x, r, w = _normal((7, 96), torch.float32, 1), _normal((7, 96), torch.float32, 2), 1 + 0.3 * _normal((96,), torch.float32, 3)
    a, b = _normal((7, 96), torch.float32, 4), _normal((7, 96), torch.float32, 5)
    y, h, rstd = N.rms_norm_forward(x, w, r, EPS, -1, 0.25, 7)
    got = N.rms_norm_backward(a, h, rstd, w, b, -1, 0.25, 7)
    _, off = ref.rms_backward(a, h, rstd, w, b, -1, 0.25, 7)
    m = ref.mask_like(x, 0.25, 7)
    f64 = lambda t: t.cpu().double()

    def f(x, r, w):
        h = r + x * m
        return ((h * ((h * h).mean(-1, keepdim=True) + EPS) ** -0.5 * w) * f64(a)).sum() + (h * f64(b)).sum()

    args = [f64(x), f64(r), f64(w)]
    for k in range(3):
        v = torch.randn(args[k].shape, generator=torch.Generator().manual_seed(10 + k), dtype=torch.float64)
        up, down = list(args), list(args)
        up[k], down[k] = args[k] + 1e-6 * v, args[k] - 1e-6 * v
        want = float(f(*up) - f(*down)) / 2e-6
        g, o = (got[0], off[0]) if k == 0 else (got[1], off[1]) if k == 1 else (got[2], off[2])
        along, bound = float((f64(g) * v).sum()), float((o * v.abs()).sum())
        # the kernel's gradient is of its fp32 h and rstd, both off by less than 8 u, so every term of the gradient by less than 32 u
        size = float((f64(g).abs() * v.abs()).sum()) + float((f64(a).abs() * f64(rstd)[:, None] * f64(w).abs()).sum())
        assert abs(along - want) <= bound + 32 * ref.U * size + 1e-7


def test_many_rows_and_planes():
    """more rows and tiles than the workgroups of the backward pass hold at once"""
    _case((20000, 72), -1, "bf16", "f32", True, 0.1)
    _case((5000, 300), -1, "f32", "f32", True, 0.0)
    _case((1500, 2048), -1, "f16", "f16", True, 0.0)
    _case((300, 20, 31, 17), 1, "f16", "f32", True, 0.1)
    _case((5, 1040, 40, 41), 1, "bf16", "f32", True, 0.1)


def test_deterministic():
    x, dy = _normal((3000, 520), torch.bfloat16, 1), _normal((3000, 520), torch.bfloat16, 2)
    y, h, rstd = N.rms_norm_forward(x)
    first = N.rms_norm_backward(dy, h, rstd)
    for _ in range(3):
        again = N.rms_norm_backward(dy, h, rstd)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("shape,axis", [((33, 100), -1), ((600, 1001), -1), ((700, 5001), -1), ((3, 40003), -1), ((3, 20, 5, 7), 1), ((2, 1100, 3, 5), 1)])
def test_in_place_through_the_abi(shape, axis):
    """outputs may be inputs of their type; what is too close is refused"""
    n = shape[axis]
    inner = 1 if axis == -1 else shape[2] * shape[3]
    d = xb.make_norm_desc(x_outer := shape[0], n, inner, "f16", "f32", EPS)
    x, r, w = _normal(shape, torch.float16, 1), _normal(shape, torch.float16, 2), _normal((n,), torch.float32, 3)
    y, h, rstd = N.rms_norm_forward(x, w, r, EPS, axis, 0.3, 5)
    drop = xb.make_drop(5, ref.q16(0.3))
    x2, r2, rstd2 = x.clone(), r.clone(), torch.empty_like(rstd)
    xb.xconv_rmsnorm_fwd(d, x2, r2, w, x2, r2, rstd2, drop)
    assert torch.equal(x2, y) and torch.equal(r2, h) and torch.equal(rstd2, rstd) and x_outer == shape[0]
    dy, dh = _normal(shape, torch.float16, 4), _normal(shape, torch.float16, 5)
    want = N.rms_norm_backward(dy, h, rstd, w, dh, axis, 0.3, 5)
    dw, ws = torch.empty_like(w), xb.alloc_bytes(xb.xconv_rmsnorm_workspace_bytes(d), DEV)
    xb.xconv_rmsnorm_bwd(d, dy, h, rstd, w, dh, dy, dh, dw, ws, drop)
    assert torch.equal(dy, want[0]) and torch.equal(dh, want[1]) and torch.equal(dw, want[2])
    with pytest.raises(xb.XConvError):
        xb.xconv_rmsnorm_fwd(d, x, r, w, y, y, rstd, drop)
    torch.cuda.synchronize()


def test_streams_and_graphs():
    """a step captured once and replayed on new data, with eager work between the replays"""
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    x, r = _normal((200, 96), torch.bfloat16, 1), _normal((200, 96), torch.bfloat16, 2)
    w = 1 + 0.3 * _normal((96,), torch.float32, 3)
    dy, dh = _normal((200, 96), torch.bfloat16, 4), _normal((200, 96), torch.bfloat16, 5)

    def one():
        y, h, rstd = N.rms_norm_forward(x, w, r, EPS, -1, 0.2, 3, step)
        return (y, h, rstd) + tuple(N.rms_norm_backward(dy, h, rstd, w, dh, -1, 0.2, 3, step))

    one()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        aside = one()
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(aside, one()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = one()
    for k in range(4):
        x.copy_(_normal((200, 96), torch.bfloat16, 20 + k))
        step.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        assert all(torch.equal(a, b) for a, b in zip(got, one()))
        torch.cuda.synchronize()


def test_places_beyond_32_bits():
    """rows whose values lie past 2^32: 65537 + 8 rows of 65536"""
    rows, n = 65545, 65536
    x = torch.zeros(rows, n, dtype=torch.bfloat16, device=DEV)
    x[-3:] = _normal((3, n), torch.bfloat16, 1)
    y, h, rstd = N.rms_norm_forward(x, None, None, EPS, -1, 0.5, 9)
    keep = torch.from_numpy(ref.kept(9, 32768, (rows - 3) * n, 3 * n)).view(3, n)
    tail = x[-3:].cpu().double() * keep * 2
    del x
    want = tail * ((tail ** 2).mean(-1, keepdim=True) + EPS) ** -0.5
    # as of token_reference: a product, the sum of squares, root, two products
    ref.close(y[-3:], want, want.abs() * ref.U * (ref.depth(n) / 2 + 20) + ref.rounding(want, torch.bfloat16))
    assert bool((y[:5] == 0).all())
    del y
    dx, dr, _ = N.rms_norm_backward(h, h, rstd, None, None, -1, 0.5, 9, need=(True, True, False))
    hs, rs = h[-3:].clone(), rstd[-3:].clone()
    small, _, _ = N.rms_norm_backward(hs, hs, rs)
    assert torch.equal(dr[-3:], small) and torch.equal(dx[-3:].cpu() == 0, (~keep) | (small.cpu() == 0))


def test_planes_beyond_32_bits():
    """maps whose values lie past 2^32; the last image against the same image alone, whose mask is moved to its place"""
    n, c, h, w = 71000, 64, 31, 31
    m = c * h * w
    x = torch.zeros(n, c, h, w, dtype=torch.bfloat16, device=DEV)
    x[-1] = _normal((c, h, w), torch.bfloat16, 1)
    keep = torch.from_numpy(ref.kept(9, 32768, (n - 1) * m, m)).view(1, c, h, w).to(DEV)
    alone = torch.where(keep, x[-1:] * 2, 0)
    y, s, rstd = N.rms_norm_forward(x, None, None, EPS, 1, 0.5, 9)
    wanted = N.rms_norm_forward(alone, None, None, EPS, 1)
    assert torch.equal(s[-1:], alone) and torch.equal(y[-1:], wanted[0]) and torch.equal(rstd.view(n, h, w)[-1:], wanted[2].view(1, h, w))
    assert not bool(y[:3].any())
    del y, s
    q, scale, _ = N.rms_norm_8bit(x, None, None, EPS, 1, torch.int8)
    small = N.rms_norm_8bit(x[-1:].clone(), None, None, EPS, 1, torch.int8)
    assert torch.equal(q[-1:], small[0]) and torch.equal(scale.view(n, h, w)[-1:], small[1].view(1, h, w))
    del q
    dx, dr, _ = N.rms_norm_backward(x, x, rstd, None, None, 1, 0.5, 9, need=(True, True, False))
    hs, rs = x[-1:].clone(), rstd.view(n, h, w)[-1:].clone()
    small = N.rms_norm_backward(hs, hs, rs, None, None, 1)[0]
    assert torch.equal(dr[-1:], small) and torch.equal(dx[-1:] == 0, ~keep | (small == 0))


def test_module():
    m = N.XRMSNorm(40, axis=1, p=0.25).to(DEV)
    x, r = _normal((2, 40, 3, 3), torch.float32, 1), _normal((2, 40, 3, 3), torch.float32, 2)
    y, h = m(x, r)
    want = N.rms_norm_forward(x, m.weight.detach(), r, 1e-6, 1, 0.25, m.last_seed)
    assert torch.equal(y, want[0]) and torch.equal(h, want[1])
    (y.sum() + h.sum()).backward()
    assert m.weight.grad is not None
    m.eval()
    y, h = m(x, r)
    assert torch.equal(h, x + r) and isinstance(m(x), torch.Tensor)
    plain = N.XRMSNorm(40, elementwise_affine=False)
    assert not list(plain.parameters())
    with pytest.raises(RuntimeError, match="40 channels"):
        m(x.permute(0, 2, 3, 1))
    m.train()
    with pytest.raises(RuntimeError, match="captured graph"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            m(x)
    torch.cuda.synchronize()


def test_refusals():
    x, w = torch.ones(4, 8, device=DEV), torch.ones(8, device=DEV)
    y, h, rstd = N.rms_norm_forward(x, w)
    for call in (lambda: N.rms_norm_forward(x, torch.ones(7, device=DEV)), lambda: N.rms_norm_forward(x, w.half()), lambda: N.rms_norm_forward(x, w.cpu()),
                 lambda: N.rms_norm_forward(x, w, x[:3]), lambda: N.rms_norm_forward(x, w, x.half()), lambda: N.rms_norm_forward(x, w, x.cpu()),
                 lambda: N.rms_norm_forward(x.double()), lambda: N.rms_norm_forward(x, axis=0), lambda: N.rms_norm_forward(x, step=torch.ones(1, device=DEV)),
                 lambda: N.rms_norm_backward(x[:3], h, rstd, w), lambda: N.rms_norm_backward(x, h, rstd[:3], w), lambda: N.rms_norm_backward(x, h, rstd, w, x[:2]),
                 lambda: N.rms_norm_backward(x, h, rstd.half(), w), lambda: N.rms_norm_8bit(x, dtype=torch.uint8), lambda: N.rms_norm_8bit(x, w, x.half()),
                 lambda: N.rms_norm_backward(x, h, rstd, param_dtype=torch.float16)):
        with pytest.raises(RuntimeError):
            call()
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(xb.XConvError):
            N.rms_norm_forward(x, w, eps=eps)
    with pytest.raises(ValueError):
        N.rms_norm_forward(x, w, p=1.5)
