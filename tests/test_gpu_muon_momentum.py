"""The momentum of a Muon step against 64 bits: M <- M + (1 - momentum)(G - M) with 1 - momentum rounded once, from 64 bits.

With u = 2^-24 the difference, the factor, the product and the sum are one rounding each: |error| <= u (3 (1 - momentum) |G - M| + |M'|),
and 2 u (1 - momentum) |G| where M is zero (the difference and the sum are exact)."""
import ctypes

import pytest
import torch

from paper_2106_06998_amd import binding as xb
from paper_2106_06998_amd import optim
from test_gpu_orth import DEV, gradient, say

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SHAPES = [(20, 33), (100, 90), (300, 900)]       # one workgroup, steps one at a time, steps in groups


@pytest.mark.parametrize("momentum", [0.0, 0.1, 0.9, 0.95, 0.99, 0.999, 0.9999, 1.0])
def test_momentum_is_as_near_as_its_roundings(momentum):
    say("muon_step, momentum", momentum, SHAPES)
    gs = [gradient(*s, 3 + i) for i, s in enumerate(SHAPES)]
    for start in (0.0, 0.3):
        ms = [start * gradient(*s, 13 + i) for i, s in enumerate(SHAPES)]
        w, g, m = ([t.to(DEV) for t in v] for v in ([torch.zeros(s) for s in SHAPES], gs, ms))
        optim.muon_step(w, g, m, 0.1, momentum)
        torch.cuda.synchronize()
        for got, g0, m0 in zip(m, gs, ms):
            g0, m0, got = g0.double(), m0.double(), got.cpu().double()
            want = m0 + (1 - momentum) * (g0 - m0)
            allowed = U * (2 * (1 - momentum) * g0.abs() if start == 0.0 else 3 * (1 - momentum) * (g0 - m0).abs() + want.abs())
            assert bool(((got - want).abs() <= 1.001 * allowed + 2.0 ** -149).all()), (momentum, start, g0.shape)


def test_both_entry_points_take_the_same_step():
    """A momentum that is a float as it stands: the step of 32-bit parameters and the one of 64-bit parameters give the same bits."""
    g = gradient(40, 70, 1).to(DEV)
    args = xb.make_orth_args()
    out = []
    for call, kind in ((xb.xconv_muon_step, xb.xconv_muon_args), (xb.xconv_muon_step64, xb.xconv_muon_args64)):
        w, m = torch.ones(40, 70, device=DEV), 0.5 * g
        items = xb.make_orth_items([(40, 70, g, w, m)])
        ws = xb.alloc_bytes(xb.xconv_orth_workspace_bytes(items, 1, args))
        call(items, 1, args, kind(0.25, 0.75, 0.5, 1), ws)
        torch.cuda.synchronize()
        out.append((w, m))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
    assert ctypes.sizeof(xb.xconv_muon_args64) == 32
