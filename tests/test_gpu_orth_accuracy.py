"""The orthogonalisation at the accuracy that its arithmetic has (orth_reference): every shape where another kernel, tile or grouping of
steps begins, and spectra that steps in groups take furthest from 64 bits.  The bounds in test_gpu_orth.py hold for any rounding; these are
a few times the error of the documented one, so that a product that loses its second fp16 numbers shows."""
import pytest
import torch

import orth_reference as ref
from paper_2106_06998_amd import optim
from test_gpu_orth import DEV, SHAPES, TD, gradient, say

pytestmark = pytest.mark.gpu

BOUNDARIES = [(64, 768), (64, 769), (65, 768), (768, 64), (769, 20), (8, 900), (33, 257), (1, 769), (64, 2000), (256, 300), (257, 300), (256, 1023), (256, 1024),
              (300, 873), (300, 874), (128, 2047), (128, 2048)]


def check(got, g, **kw):
    want, norm, _ = ref.tolerances(g, **kw)
    off = float(torch.linalg.vector_norm(got.to(want.device).double() - want))
    assert off <= norm, (off, norm, off / float(torch.linalg.vector_norm(want)))


@pytest.mark.parametrize("rows,cols", SHAPES + BOUNDARIES)
def test_every_shape_in_fp32(rows, cols):
    say("orthogonalize, accuracy", rows, cols)
    g = gradient(rows, cols, rows + 3 * cols)
    o = optim.orthogonalize(g.to(DEV))
    torch.cuda.synchronize()
    check(o, g)


@pytest.mark.parametrize("rows,cols", [(16, 144), (64, 576), (576, 64), (64, 769), (200, 147), (147, 200), (320, 320), (300, 900), (900, 300)])
def test_muon_from_zero_in_fp32(rows, cols):
    """W = 0, lr = 1: W becomes the update itself."""
    g = gradient(rows, cols, 5)
    say("muon_step from zero, accuracy", rows, cols)
    w, m = torch.zeros(rows, cols, device=DEV), torch.zeros(rows, cols, device=DEV)
    optim.muon_step([w], [g.to(DEV)], [m], lr=1.0, momentum=0.0, nesterov=False)
    torch.cuda.synchronize()
    check(-w / max(1.0, rows / cols) ** 0.5, g)


@pytest.mark.parametrize("way", sorted(ref.WAYS))
def test_every_way_in_fp32_and_the_same_bits_alone(way):
    shapes, _ = ref.WAYS[way]
    say("orthogonalize", way, shapes[0], "x", len(shapes))
    gs = [gradient(*s, 7 + i).to(DEV) for i, s in enumerate(shapes)]
    many = optim.orthogonalize(gs)
    torch.cuda.synchronize()
    for k in sorted({0, len(shapes) - 1}):
        check(many[k], gs[k])            # (the reference on the device, too)
        alone = optim.orthogonalize(gs[k])
        torch.cuda.synchronize()
        assert torch.equal(alone, many[k])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("way", [w for w in sorted(ref.WAYS) if w.startswith("groups")] + ["steps, split sums", "steps, tiles of 128"])
def test_sixteen_bits_in_large_tiles_groups_and_split_sums(way, dtype):
    shapes, _ = ref.WAYS[way]
    say("orthogonalize and muon_step", way, dtype)
    gs = [gradient(*s, 17 + i, dtype).to(DEV) for i, s in enumerate(shapes)]
    many = optim.orthogonalize(gs)
    ws = [torch.zeros_like(g) for g in gs]
    optim.muon_step(ws, gs, [torch.zeros_like(g, dtype=torch.float32) for g in gs], lr=1.0, momentum=0.0, nesterov=False)
    torch.cuda.synchronize()
    k = len(shapes) - 1
    want, _, each = ref.tolerances(gs[k])
    scale = max(1.0, shapes[k][0] / shapes[k][1]) ** 0.5
    assert ref.excess(many[k], want, TD[dtype], each) <= each
    assert ref.excess(ws[k], -scale * want, TD[dtype], scale * each) <= scale * each


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 7])
@pytest.mark.parametrize("coef", [ref.COEF, (1.875, -1.25, 0.375)])
def test_groups_of_any_number_of_steps(steps, coef):
    from paper_2106_06998_amd import binding as xb

    for shape in ((300, 900), (1000, 290)):
        say("orthogonalize, accuracy", shape, steps, coef)
        g = gradient(*shape, 3 * steps)
        sizes = xb.xconv_orth_plan_info(xb.make_orth_items([(*shape, None, None, None)]), 1, xb.make_orth_args(steps=steps, coefficients=coef))["groups"]
        o = optim.orthogonalize(g.to(DEV), steps, coef)
        torch.cuda.synchronize()
        check(o, g, steps=steps, coef=coef, sizes=sizes)


def spectrum(name, rows, cols):
    """Matrices that take the steps' errors further than a gradient does."""
    gen = torch.Generator().manual_seed(len(name))
    m = min(rows, cols)
    noise = torch.randn(rows, cols, generator=gen, dtype=torch.float64)
    if name == "one column" or name == "one row":
        noise[:, 3:4] *= 1e3 if name == "one column" else 1.0
        noise[3:4] *= 1e3 if name == "one row" else 1.0
        return noise.float()
    u, _, v = torch.linalg.svd(noise, full_matrices=False)
    s = torch.ones(m, dtype=torch.float64)
    if name.startswith("falls to"):
        s = torch.logspace(0, float(name.split("-")[1]) * -1, m, dtype=torch.float64)
    elif name == "one large value":
        s[1:] = 0.1
    elif name == "half of the rank":
        s[m // 2:] = 0.0
    else:
        assert name == "all alike"
    return ((u * s) @ v).float()


@pytest.mark.parametrize("name", ["falls to 1e-2", "falls to 1e-3", "falls to 1e-4", "one large value", "half of the rank", "all alike", "one column", "one row"])
@pytest.mark.parametrize("rows,cols", [(48, 100), (64, 800), (200, 147), (320, 330), (384, 900), (900, 384)])
def test_spectra(name, rows, cols):
    g = spectrum(name, rows, cols)
    o = optim.orthogonalize(g.to(DEV))
    torch.cuda.synchronize()
    want = ref.exact(g)
    single = ref.documented(g, sizes=[1] * 5).double() - want
    size = float(torch.linalg.vector_norm(want))
    say("spectrum", name, rows, cols, "off %.2e, one step at a time on the CPU %.2e" % (float(torch.linalg.vector_norm(o.cpu().double() - want)) / size,
                                                                                        float(torch.linalg.vector_norm(single)) / size))
    check(o, g)
