"""The reference of the orthogonalisation's accuracy tests, on the CPU: the documented arithmetic is at the level of fp32 products, and its
tolerances notice a last product of 11 bits in every type, at every shape that the GPU tests take."""
import ctypes

import pytest
import torch

import orth_reference as ref
from paper_2106_06998_amd import binding as xb

SHAPES = [(1, 1), (2, 2), (16, 144), (64, 576), (65, 768), (130, 200), (300, 400), (300, 900), (1100, 260)]


def matrix(rows, cols, seed):
    return torch.randn(rows, cols, generator=torch.Generator().manual_seed(seed)) * 1e-3


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_documented_arithmetic_is_near_fp32(rows, cols):
    g = matrix(rows, cols, 1)
    want, norm, each = ref.tolerances(g)
    size = float(torch.linalg.vector_norm(want))
    assert 2.0 ** -20 * size <= norm <= 4e-5 * size
    assert float((ref.documented(g).double() - want).abs().max()) <= each


@pytest.mark.parametrize("rows,cols", [s for s in SHAPES if min(s) > 1])
def test_a_last_product_of_eleven_bits_is_noticed(rows, cols):
    g = matrix(rows, cols, 2)
    want, norm, each = ref.tolerances(g)
    off = ref.documented(g, last_numbers=1)
    assert float(torch.linalg.vector_norm(off.double() - want)) > norm
    if rows * cols >= 10000:          # enough elements for some to lie next to a rounding's boundary
        for dtype in (torch.bfloat16, torch.float16):
            assert ref.excess(ref.documented(g).to(dtype), want, dtype, each) <= each
            assert ref.excess(off.to(dtype), want, dtype, each) > each


def test_half_a_place():
    for dtype in (torch.bfloat16, torch.float16):
        v = torch.tensor([1.0, 1.5, 0.3, 3.9, 2.0 ** -20, 0.0, 60000.0], dtype=torch.float64)
        for x in v.tolist():
            near = torch.tensor(x, dtype=torch.float64)
            r = near.to(dtype)
            assert abs(float(r) - x) <= float(ref.half_place(near, dtype))
    assert float(ref.half_place(torch.tensor(1.0), torch.bfloat16)) == 2.0 ** -8 and float(ref.half_place(torch.tensor(1.0), torch.float16)) == 2.0 ** -11
    assert float(ref.half_place(torch.tensor(0.0), torch.float16)) == 2.0 ** -25


def test_groups():
    assert ref.groups(512, 4608, 5) == [3, 2] and ref.groups(512, 1000, 5) == [1] * 5 and ref.groups(362, 725, 6) == [3, 2, 1] and ref.groups(127, 9000, 2) == [1, 1]


def plan(shapes, index=0, steps=5):
    items = xb.make_orth_items([(r, c, None, None, None) for r, c in shapes])
    return xb.xconv_orth_plan_info(items, len(shapes), xb.make_orth_args(steps=steps), index)


@pytest.mark.parametrize("way", sorted(ref.WAYS))
def test_calls_take_the_way_that_they_are_tested_for(way):
    shapes, expected = ref.WAYS[way]
    for index in (0, len(shapes) - 1):
        p = plan(shapes, index)
        groups = p.pop("groups")
        assert p == {**{k: 0 for k in xb.ORTH_PLAN_FIELDS}, **expected}
        assert groups == ref.groups(*shapes[index], 5) and (groups == [3, 2]) == (expected["kind"] == ref.GROUPED)


def test_groups_of_the_library_are_those_of_the_reference():
    for shape in ((127, 5000), (128, 2047), (128, 2048), (300, 873), (300, 874), (512, 1023), (512, 1024), (4096, 700), (1, 1), (64, 768)):
        for steps in (0, 1, 2, 3, 4, 5, 7):
            assert plan([shape], 0, steps)["groups"] == ref.groups(*shape, steps), (shape, steps)


def test_plan_statuses():
    args, out = xb.make_orth_args(), (ctypes.c_int32 * 16)()
    items = xb.make_orth_items([(4, 4, None, None, None)])
    ask = lambda it, n, a, k, o: xb.lib().xconv_orth_plan_info(it, n, a, k, o)
    assert ask(items, 1, ctypes.byref(args), 0, out) == xb.XCONV_OK
    assert ask(items, 1, ctypes.byref(args), 1, out) == xb.XCONV_EINVAL and ask(items, 1, ctypes.byref(args), -1, out) == xb.XCONV_EINVAL
    assert ask(items, 1, ctypes.byref(args), 0, None) == xb.XCONV_EINVAL and ask(items, 1, None, 0, out) == xb.XCONV_EINVAL
    assert ask(items, 0, ctypes.byref(args), 0, out) == xb.XCONV_EINVAL
