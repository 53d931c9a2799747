"""Orthogonalisation and the Muon step (xconv_orth, xconv_muon_step, optim.py) against their definition in 64 bits.

The tolerance of a case is computed from its exact iterates before anything is compared.  A step's products have operands of 22
bits (relative error at most 2^-22 a product of two) and fp32 sums of K terms in runs of 16 (an error that grows as the square root
of their number: 2^-24 sqrt(K / 16)); with eps = 2^-22 + 2^-24 sqrt(K / 16) step k puts an error of at most
(|a| + 3 |b| s^2 + 5 |c| s^4) eps |X_k|_F into X, s being the largest singular value of X_k, and every later step multiplies an
error by at most L, the largest slope of s (a + b s^2 + c s^4) over the range the singular values reach."""
import math

import numpy as np
import pytest
import torch

from paper_2106_06998_amd import binding as xb
from paper_2106_06998_amd import optim

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TD = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UOUT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
COEF = (3.4445, -4.7750, 2.0315)


def say(*a):
    print("[gpu-case]", *a, flush=True)


def exact_orth(g, steps=5, coef=COEF, eps=1e-7):
    """(O, bound of |error|_F) of a matrix of 64-bit numbers on the CPU."""
    a, b, c = coef
    x = g / max(np.linalg.norm(g), eps)
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    tops, inject = [], []
    K = max(x.shape)
    e = 2.0 ** -22 + 2.0 ** -24 * math.sqrt(K / 16)
    for _ in range(steps):
        top = float(np.linalg.norm(x, 2)) if x.size else 0.0
        tops.append(top)
        inject.append((abs(a) + 3 * abs(b) * top ** 2 + 5 * abs(c) * top ** 4) * e * np.linalg.norm(x))
        s = x @ x.T
        x = a * x + (b * s + c * (s @ s)) @ x
    s = np.linspace(0, max(tops + [1e-3]) * 1.01, 400)
    L = max(1.0, float(np.abs(a + 3 * b * s ** 2 + 5 * c * s ** 4).max()), float(np.abs(a + b * s ** 2 + c * s ** 4).max()))
    bound = sum(v * L ** (steps - 1 - k) for k, v in enumerate(inject)) + 2.0 ** -22 * L ** steps
    return (x.T if tall else x), bound


def gradient(rows, cols, seed, dtype="f32", scale=1e-3):
    rng = np.random.default_rng(seed)
    k = max(1, min(rows, cols) // 4)
    fall = np.exp(np.linspace(0.0, -2.0, k)) / math.sqrt(k)
    g = scale * ((rng.standard_normal((rows, k)) * fall) @ rng.standard_normal((k, cols)) + 0.2 * rng.standard_normal((rows, cols)))
    return torch.from_numpy(g.astype(np.float32)).to(TD[dtype])


def check_orth(got, g, dtype, **kw):
    want, bound = exact_orth(g.double().numpy(), **kw)
    got = got.detach().cpu().double().numpy()
    size = np.linalg.norm(want)
    off = np.linalg.norm(got - want)
    assert off <= bound + UOUT[dtype] * (size + bound) + 1e-30, (off, bound, size)
    return off / size if size else off


SHAPES = [(1, 1), (1, 2), (2, 1), (1, 500), (500, 1), (2, 2), (3, 5), (16, 16), (16, 144), (31, 33), (32, 64), (63, 65), (64, 64), (64, 576), (65, 64), (576, 64),
          (100, 37), (128, 128), (129, 127), (128, 1152), (200, 147), (256, 128), (130, 1000), (257, 513), (320, 320)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_one_matrix(rows, cols, dtype):
    say("orthogonalize", rows, cols, dtype)
    g = gradient(rows, cols, rows * 7 + cols, dtype)
    o = optim.orthogonalize(g.to(DEV))
    torch.cuda.synchronize()
    assert o.shape == g.shape and o.dtype == g.dtype
    check_orth(o, g, dtype)


@pytest.mark.parametrize("rows,cols", [(512, 4608), (1024, 1024), (1000, 1500), (700, 3001)])
def test_large_matrices(rows, cols):
    say("orthogonalize", rows, cols)
    g = gradient(rows, cols, 3)
    o = optim.orthogonalize(g.to(DEV))
    torch.cuda.synchronize()
    off = check_orth(o, g, "f32")
    assert off <= 1e-5          # of the order of fp32 products


@pytest.mark.parametrize("steps", [0, 1, 2, 3, 6])
def test_number_of_steps(steps):
    for shape in ((40, 90), (130, 70)):
        g = gradient(*shape, 11 + steps)
        o = optim.orthogonalize(g.to(DEV), steps)
        torch.cuda.synchronize()
        check_orth(o, g, "f32", steps=steps)


@pytest.mark.parametrize("coef", [(1.5, -0.5, 0.0), (1.875, -1.25, 0.375), (2.0, -1.5, 0.5), (1.0, 0.0, 0.0)])
def test_other_coefficients(coef):
    g = gradient(70, 150, 5)
    for steps in (4, 12):
        o = optim.orthogonalize(g.to(DEV), steps, coef)
        torch.cuda.synchronize()
        check_orth(o, g, "f32", steps=steps, coef=coef)


def test_scales_from_tiny_to_huge():
    for scale in (1e-30, 1e-12, 1.0, 1e12, 1e30):
        g = gradient(48, 100, 9, scale=scale)
        o = optim.orthogonalize(g.to(DEV), eps=0.0)
        torch.cuda.synchronize()
        check_orth(o, g, "f32", eps=0.0)
    g = gradient(48, 100, 9, scale=1e-12)        # below eps: divided by eps only
    o = optim.orthogonalize(g.to(DEV))
    torch.cuda.synchronize()
    check_orth(o, g, "f32")


def test_wide_ranges_within_a_matrix():
    """One row a million times the others, and a matrix of rank one."""
    g = gradient(40, 80, 1)
    g[3] *= 1e6
    o = optim.orthogonalize(g.to(DEV))
    torch.cuda.synchronize()
    check_orth(o, g, "f32")
    g = torch.outer(torch.linspace(-1, 1, 50), torch.linspace(0.5, 2, 70))
    o = optim.orthogonalize(g.to(DEV))
    torch.cuda.synchronize()
    check_orth(o, g, "f32")


def test_zero_and_non_finite_matrices():
    gs = [gradient(33, 70, 1), torch.zeros(33, 70), gradient(70, 33, 2), gradient(20, 20, 3)]
    gs[2][5, 6] = float("nan")
    gs[3][7, 1] = float("inf")
    for eps in (1e-7, 0.0):
        o = optim.orthogonalize([g.to(DEV) for g in gs], eps=eps)
        torch.cuda.synchronize()
        check_orth(o[0], gs[0], "f32", eps=eps)
        assert not o[1].any()
        assert torch.isnan(o[2]).all() and torch.isnan(o[3]).all()


def test_many_matrices_of_any_shape_in_one_call():
    """More than one launch holds; equal to one call each, bit for bit, whatever else is in the call."""
    shapes = [(16, 144), (64, 576), (3, 200), (200, 3), (65, 65), (128, 64), (1, 9), (40, 40)] * 8 + [(256, 300)]
    gs = [gradient(r, c, i).to(DEV) for i, (r, c) in enumerate(shapes)]
    many = optim.orthogonalize(gs)
    torch.cuda.synchronize()
    assert len(many) == len(gs)
    for i in range(0, len(gs), 5):
        one = optim.orthogonalize(gs[i])
        torch.cuda.synchronize()
        assert torch.equal(one, many[i]), shapes[i]
        check_orth(many[i], gs[i].cpu(), "f32")
    again = optim.orthogonalize(gs)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(many, again))


def test_views_weights_and_mixed_types():
    g = gradient(48, 27 * 9, 4)
    conv = g.view(48, 27, 3, 3).to(DEV)
    want = optim.orthogonalize(g.to(DEV))
    assert torch.equal(optim.orthogonalize(conv).view(48, -1), want)
    cl = conv.contiguous(memory_format=torch.channels_last)
    o = optim.orthogonalize(cl)
    torch.cuda.synchronize()
    assert o.shape == cl.shape
    check_orth(o.reshape(48, -1), g, "f32")
    wide = torch.zeros(48, 300, device=DEV)
    wide[:, 13:13 + 243] = g.to(DEV)
    assert torch.equal(optim.orthogonalize(wide[:, 13:13 + 243]), want)
    o = optim.orthogonalize(g.to(DEV).t())
    torch.cuda.synchronize()
    check_orth(o, g.t(), "f32")
    off = torch.zeros(48 * 243 + 1, dtype=torch.float16, device=DEV)
    off[1:] = g.half().reshape(-1).to(DEV)
    mixed = optim.orthogonalize([g.to(DEV), g.bfloat16().to(DEV), off[1:].view(48, 243), torch.zeros(0, 5, device=DEV)])
    torch.cuda.synchronize()
    assert [t.dtype for t in mixed[:3]] == [torch.float32, torch.bfloat16, torch.float16] and mixed[3].shape == (0, 5)
    check_orth(mixed[0], g, "f32")
    check_orth(mixed[1], g.bfloat16(), "bf16")
    check_orth(mixed[2], g.half(), "f16")


def muon_reference(w, g, m, lr, mu, decay, nesterov):
    w, g, m = (t.double().numpy() for t in (w, g, m))
    m1 = m + (1 - mu) * (g - m)
    u = g + mu * (m1 - g) if nesterov else m1
    o, bound = exact_orth(u.reshape(u.shape[0], -1))
    rows, cols = o.shape
    s = lr * math.sqrt(max(1.0, rows / cols))
    return (1 - lr * decay) * w - s * o.reshape(w.shape), m1, s * (bound + 3e-7 * np.linalg.norm(o))


@pytest.mark.parametrize("dtype,gtype", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16")])
@pytest.mark.parametrize("nesterov", [True, False])
def test_muon_step(dtype, gtype, nesterov):
    shapes = [(16, 9, 4, 4), (64, 64, 3, 3), (40, 10), (10, 40), (1, 7), (300, 200), (130, 65, 1, 1)]
    ws = [(gradient(s[0], int(np.prod(s[1:])), i, scale=1.0) * 0.1).view(s).to(TD[dtype]) for i, s in enumerate(shapes)]
    gs = [gradient(s[0], int(np.prod(s[1:])), 50 + i).view(s).to(TD[gtype]) for i, s in enumerate(shapes)]
    ms = [gradient(s[0], int(np.prod(s[1:])), 90 + i, scale=3e-4).view(s) for i, s in enumerate(shapes)]
    wd, gd, md = ([t.to(DEV) for t in v] for v in (ws, gs, ms))
    lr, mu, decay = 0.05, 0.9, 0.1
    optim.muon_step(wd, gd, md, lr, mu, decay, nesterov)
    torch.cuda.synchronize()
    for w, g, m, a, b, c in zip(ws, gs, ms, wd, gd, md):
        want, m1, bound = muon_reference(w, g, m, lr, mu, decay, nesterov)
        off = np.abs(a.cpu().double().numpy() - want)
        # the step's own error, two roundings of the sum in fp32 and one to the type of the weights
        tol = bound + (UOUT[dtype] + 3 * 2.0 ** -24) * np.linalg.norm(want) + (1e-7 if dtype == "f16" else 0)
        assert np.linalg.norm(off) <= tol, (w.shape, np.linalg.norm(off), tol)
        assert np.all(np.abs(c.cpu().double().numpy() - m1) <= 4 * 2.0 ** -24 * (np.abs(m1) + np.abs(g.double().numpy()) + np.abs(m.double().numpy())))
        assert torch.equal(b.cpu(), g)


def test_muon_step_on_other_orders_of_memory():
    w0, g0, m0 = (gradient(24, 20 * 9, 7 + i, scale=0.1).view(24, 20, 3, 3).to(DEV) for i in range(3))
    want_w, want_m = w0.clone(), m0.clone()
    optim.muon_step([want_w], [g0], [want_m], 0.1)
    for wf, gf, mf in ((torch.channels_last, torch.channels_last, torch.channels_last), (torch.channels_last, torch.contiguous_format, torch.contiguous_format),
                       (torch.contiguous_format, torch.channels_last, torch.channels_last)):
        w, g, m = w0.clone(memory_format=wf), g0.clone(memory_format=gf), m0.clone(memory_format=mf)
        optim.muon_step([w], [g], [m], 0.1)
        torch.cuda.synchronize()
        assert float((w - want_w).abs().max()) <= 1e-6 and torch.equal(m, want_m)
    big = torch.zeros(24, 40, 3, 3, device=DEV)
    big[:, ::2] = w0
    w, m = big[:, ::2], m0.clone()
    optim.muon_step([w], [g0], [m], 0.1)
    torch.cuda.synchronize()
    assert torch.equal(w, want_w) and not big[:, 1::2].any()


def test_optimiser_trains_and_counts_versions():
    torch.manual_seed(0)
    lin = torch.nn.Linear(40, 24, bias=False, device=DEV)
    target = torch.randn(24, 40, device=DEV)
    x = torch.randn(200, 40, device=DEV)
    opt = optim.Muon(lin.parameters(), lr=0.1, momentum=0.9)
    first = None
    for _ in range(60):
        opt.zero_grad()
        loss = ((lin(x) - x @ target.t()) ** 2).mean()
        loss.backward()
        before = lin.weight._version
        opt.step()
        assert lin.weight._version > before
        first = float(loss) if first is None else first
    assert float(loss) < 0.2 * first
    state = opt.state_dict()
    assert state["state"][0]["momentum_buffer"].dtype == torch.float32
    # a tensor that a graph still needs is known to have changed
    w = torch.randn(5, 6, device=DEV, requires_grad=True)
    y = (w * w).sum()
    with torch.no_grad():
        optim.muon_step([w.detach()], [torch.ones(5, 6, device=DEV)], [torch.zeros(5, 6, device=DEV)], 0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_on_a_side_stream_and_in_a_graph():
    gs = [gradient(r, c, i).to(DEV) for i, (r, c) in enumerate([(64, 100), (33, 20), (200, 90)])]
    want = optim.orthogonalize(gs)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = optim.orthogonalize(gs)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ws = [0.1 * g.clone() * 1e3 for g in gs]
    ms = [torch.zeros_like(g) for g in gs]
    w2, m2 = [w.clone() for w in ws], [m.clone() for m in ms]
    start_w, start_m = [w.clone() for w in ws], [m.clone() for m in ms]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        optim.muon_step(ws, gs, ms, 0.05)
    for t, u in zip(ws + ms, start_w + start_m):
        t.copy_(u)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        optim.muon_step(w2, gs, m2, 0.05)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ws + ms, w2 + m2))
        gs[0].mul_(1.5)


def test_outputs_lie_only_where_they_should():
    """Guard values around O, W and M through the C ABI, at odd extents and an odd offset."""
    rows, cols = 37, 83
    n = rows * cols
    g = gradient(rows, cols, 1)
    G = torch.full((n + 7,), 5.0, device=DEV)
    G[3:3 + n] = g.reshape(-1).to(DEV)
    O = torch.full((n + 7,), 5.0, device=DEV)
    M = torch.full((n + 7,), 5.0, device=DEV)
    M[3:3 + n] = 0
    args = xb.make_orth_args()
    items = xb.make_orth_items([(rows, cols, G[3:], O[3:], M[3:])])
    size = xb.xconv_orth_workspace_bytes(items, 1, args)
    ws = torch.full((size + 256,), 77, dtype=torch.uint8, device=DEV)
    xb.xconv_orth(items, 1, args, ws[:size])
    torch.cuda.synchronize()
    assert (ws[size:] == 77).all() and (O[:3] == 5).all() and (O[-4:] == 5).all()
    check_orth(O[3:3 + n].view(rows, cols), g, "f32")
    xb.xconv_muon_step(items, 1, args, xb.xconv_muon_args(0.1, 0.9, 0.0, 1), ws[:size])
    torch.cuda.synchronize()
    for t in (O, M, G):
        assert (t[:3] == 5).all() and (t[-4:] == 5).all()
    assert (ws[size:] == 77).all() and float(M[3:3 + n].abs().max()) < 1


def test_refusals_on_the_device():
    g = gradient(8, 9, 1).to(DEV)
    with pytest.raises(RuntimeError, match="not supported"):
        optim.orthogonalize(g.double())
    with pytest.raises(RuntimeError, match="matrices"):
        optim.orthogonalize(g[0])
    with pytest.raises(xb.XConvError):
        optim.orthogonalize(g, coefficients=(9.0, 0.0, 0.0))
    with pytest.raises(xb.XConvError):
        optim.orthogonalize(g, steps=65)
    with pytest.raises(xb.XConvError):
        optim.orthogonalize(g, steps=-1)
    with pytest.raises(xb.XConvError):
        optim.orthogonalize(g, eps=float("nan"))
    w, m = g.clone(), torch.zeros_like(g)
    with pytest.raises(RuntimeError, match="another shape"):
        optim.muon_step([w], [g[:4]], [m], 0.1)
    with pytest.raises(RuntimeError, match="float32"):
        optim.muon_step([w], [g], [m.half()], 0.1)
    with pytest.raises(RuntimeError, match="as many"):
        optim.muon_step([w], [g, g], [m], 0.1)
    with pytest.raises(xb.XConvError):
        optim.muon_step([w], [g], [m], float("inf"))
    torch.cuda.synchronize()
    assert torch.equal(w, g) and not m.any()


@pytest.mark.parametrize("rows,cols", [(64, 768), (64, 769), (65, 768), (768, 64), (769, 20), (8, 900), (33, 257), (1, 769), (64, 2000)])
def test_where_small_matrices_end(rows, cols):
    """Around the extents up to which a matrix is one workgroup's."""
    for dtype in ("f32", "f16"):
        g = gradient(rows, cols, rows + cols, dtype)
        o = optim.orthogonalize(g.to(DEV))
        torch.cuda.synchronize()
        check_orth(o, g, dtype)


@pytest.mark.parametrize("rows,cols", [(256, 2304), (96, 3200), (1100, 1300), (1088, 2100)])
def test_split_sums(rows, cols):
    say("orthogonalize", rows, cols)
    g = gradient(rows, cols, 5, "bf16")
    o = optim.orthogonalize(g.to(DEV))
    torch.cuda.synchronize()
    check_orth(o, g, "bf16")


@pytest.mark.parametrize("shape", [(256, 1152), (512, 1600), (130, 700), (120, 2000)])
def test_larger_tiles_give_the_same_bits(shape):
    """Enough equal matrices are taken in larger tiles: not one bit of a result depends on it."""
    say("orthogonalize", shape, "alone and among others")
    gs = [gradient(*shape, i).to(DEV) for i in range(20)]
    many = optim.orthogonalize(gs)
    torch.cuda.synchronize()
    for i in (0, 7, 19):
        one = optim.orthogonalize(gs[i])
        torch.cuda.synchronize()
        assert torch.equal(one, many[i])
    check_orth(many[3], gs[3].cpu(), "f32")


def test_muon_on_large_layers():
    say("muon_step 6 x 300 x 1300")
    ws = [gradient(300, 1300, i, scale=1.0) * 0.1 for i in range(6)]
    gs = [gradient(300, 1300, 50 + i) for i in range(6)]
    for dtype in ("f32", "bf16"):
        wd = [w.to(TD[dtype]).to(DEV) for w in ws]
        gd = [g.to(TD[dtype]).to(DEV) for g in gs]
        md = [torch.zeros(300, 1300, device=DEV) for _ in ws]
        optim.muon_step(wd, gd, md, 0.05, 0.9, 0.1)
        torch.cuda.synchronize()
        want, m1, bound = muon_reference(ws[2].to(TD[dtype]), gs[2].to(TD[dtype]), torch.zeros(300, 1300), 0.05, 0.9, 0.1, True)
        off = np.linalg.norm(wd[2].cpu().double().numpy() - want)
        assert off <= bound + (UOUT[dtype] + 3 * 2.0 ** -24) * np.linalg.norm(want)


# ---- steps in groups: the next A from this one (matrices of more than 256 rows that are at least twice as wide) ---------------
def group_bound(g, steps, coef, eps=1e-7):
    """The bound above where every step's A may come from the one before it: an error of A grows by at most
    G = max |d (l q(l)^2) / dl| a step, and at most two steps lie between X X^T and the A that is used."""
    a, b, c = coef
    want, bound = exact_orth(g, steps, coef, eps)
    l = np.linspace(0, 1.3, 400)
    q, slope = a + b * l + c * l * l, b + 2 * c * l
    grow = max(1.0, float(np.abs(q * q + 2 * l * q * slope).max()))
    return want, bound * 3 * grow ** 2


@pytest.mark.parametrize("shape", [(257, 514), (514, 257), (300, 1500), (390, 781)])
@pytest.mark.parametrize("steps,coef", [(1, COEF), (2, COEF), (3, COEF), (4, COEF), (5, COEF), (6, COEF), (7, COEF), (9, (1.875, -1.25, 0.375)), (6, (1.5, -0.5, 0.0))])
def test_steps_in_groups(shape, steps, coef):
    say("orthogonalize", shape, steps, coef)
    g = gradient(*shape, 5 + steps)
    o = optim.orthogonalize(g.to(DEV), steps, coef)
    torch.cuda.synchronize()
    want, bound = group_bound(g.double().numpy(), steps, coef)
    off = np.linalg.norm(o.cpu().double().numpy() - want)
    size = np.linalg.norm(want)
    assert off <= bound + 2.0 ** -24 * size
    assert off <= 2e-5 * size       # a large matrix' bound says little: of the order of fp32 products


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_groups_of_sixteen_bits(dtype):
    for shape in ((260, 600), (600, 260)):
        say("orthogonalize", shape, dtype)
        g = gradient(*shape, 8, dtype)
        o = optim.orthogonalize(g.to(DEV))
        torch.cuda.synchronize()
        want, bound = group_bound(g.double().numpy(), 5, COEF)
        size = np.linalg.norm(want)
        assert np.linalg.norm(o.cpu().double().numpy() - want) <= min(bound, 2e-5 * size) + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -11) * size


def test_groups_beside_single_steps():
    """A list of both kinds and of small matrices: the same bits as alone, in any order."""
    shapes = [(300, 700), (64, 90), (300, 400), (1000, 270), (130, 900), (257, 514)]
    gs = [gradient(*s, 40 + i).to(DEV) for i, s in enumerate(shapes)]
    many = optim.orthogonalize(gs)
    turned = optim.orthogonalize(gs[::-1])[::-1]
    torch.cuda.synchronize()
    for i, g in enumerate(gs):
        one = optim.orthogonalize(g)
        torch.cuda.synchronize()
        assert torch.equal(one, many[i]) and torch.equal(one, turned[i]), shapes[i]


@pytest.mark.parametrize("shape,dtype", [((70, 4000), "f32"), ((4000, 70), "bf16"), ((200, 1400), "f16"), ((256, 1100), "f32"), ((300, 900), "f16"), ((1025, 2100), "f32")])
def test_groups_of_few_and_of_many_rows(shape, dtype):
    say("orthogonalize", shape, dtype)
    g = gradient(*shape, 9, dtype)
    o = optim.orthogonalize(g.to(DEV))
    torch.cuda.synchronize()
    want, bound = group_bound(g.double().numpy(), 5, COEF)
    size = np.linalg.norm(want)
    assert np.linalg.norm(o.cpu().double().numpy() - want) <= min(bound, 2e-5 * size) + UOUT[dtype] * size


KINDS = [(300, 900), (64, 90), (130, 200), (16, 144), (600, 500), (64, 4200)]


def kinds_alone(seed):
    """Weights, gradients and momenta of all kinds of matrices, and the step of each by itself."""
    g = [gradient(*s, seed + i).to(DEV) for i, s in enumerate(KINDS)]
    w = [0.1 * torch.ones_like(t) for t in g]
    m = [0.5 * t for t in g]
    one = [(a.clone(), b.clone()) for a, b in zip(w, m)]
    for (a, b), t in zip(one, g):
        optim.muon_step([a], [t], [b], lr=0.02)
    torch.cuda.synchronize()
    return w, g, m, one


def test_kinds_beside_each_other_follow_the_stream():
    """What the call reads is made just before it on its stream, and what it writes is used just after it."""
    w, g, m, one = kinds_alone(60)
    say("muon_step, kinds", KINDS)
    side = torch.cuda.Stream()
    slow = torch.ones(2048, 2048, device=DEV)
    torch.cuda.synchronize()
    for turn in range(8):
        with torch.cuda.stream(side):
            made = [torch.zeros_like(t) for t in g]
            for _ in range(3):
                slow = slow @ slow * (1.0 / 2048)
            for a, b in zip(made, g):
                a.copy_(b)
            ws, ms = [t.clone() for t in w], [t.clone() for t in m]
            optim.muon_step(ws, made, ms, lr=0.02)
            for t in made:
                t.fill_(float("nan"))
            got = [(a.clone(), b.clone()) for a, b in zip(ws, ms)]
            for t in ws + ms:
                t.fill_(float("nan"))
        side.synchronize()
        assert all(torch.equal(a, c) and torch.equal(b, d) for (a, b), (c, d) in zip(got, one)), turn


def test_kinds_in_a_graph_and_eager_calls_between():
    w, g, m, one = kinds_alone(70)
    say("muon_step in a graph, kinds", KINDS)
    ws, ms = [t.clone() for t in w], [t.clone() for t in m]
    optim.muon_step(ws, g, ms, lr=0.02)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        optim.muon_step(ws, g, ms, lr=0.02)
    for turn in range(4):
        for a, b in zip(ws + ms, w + m):
            a.copy_(b)
        graph.replay()
        w2, m2 = [t.clone() for t in w], [t.clone() for t in m]
        optim.muon_step(w2, g, m2, lr=0.02)
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) and torch.equal(b, d) for a, b, (c, d) in zip(ws, ms, one)), turn
        assert all(torch.equal(a, c) and torch.equal(b, d) for a, b, (c, d) in zip(w2, m2, one)), turn


def test_kinds_from_several_threads():
    import threading

    w, g, m, one = kinds_alone(80)
    say("muon_step from three threads, kinds", KINDS)
    good = [None] * 3

    def work(k):
        with torch.cuda.stream(torch.cuda.Stream()) as _:
            s = torch.cuda.current_stream()
            same = True
            for _ in range(6):
                ws, ms = [t.clone() for t in w], [t.clone() for t in m]
                optim.muon_step(ws, g, ms, lr=0.02)
                s.synchronize()
                same = same and all(torch.equal(a, c) and torch.equal(b, d) for a, b, (c, d) in zip(ws, ms, one))
            good[k] = same

    threads = [threading.Thread(target=work, args=(k,)) for k in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert good == [True] * 3
