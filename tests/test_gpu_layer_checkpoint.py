"""Weight gradients under activation checkpointing: the pass that is run again probes with the matrix that the estimate goes by."""
import pytest
import torch
from torch.utils.checkpoint import checkpoint

from paper_2106_06998_amd import layer as L
from paper_2106_06998_amd.dropout import XDropout

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


@pytest.mark.parametrize("reentrant", [False, True])
@pytest.mark.parametrize("mode,engine", [(m, e) for m in L.MODES for e in ("library", "framework")] + [("volume", None)])
def test_gradients(mode, engine, reentrant, monkeypatch):
    """Two layers and dropout in one checkpoint, a third layer in another: the same gradients as without, from the same state of the
    generator (the reentrant kind's first pass runs without gradients)."""
    monkeypatch.setattr(L, "_calls", L._Seeds())
    torch.manual_seed(3)
    if mode == "volume":
        make, size = lambda a, b: L.XConv3d(a, b, 3, r=4, padding=1, base_seed=a), (2, 8, 4, 6, 6)
    else:
        make, size = lambda a, b: L.XConv2d(a, b, 3, r=4, padding=1, mode=mode, engine=engine, base_seed=a), (3, 8, 7, 9)
    parts = [torch.nn.Sequential(make(8, 12), torch.nn.Tanh(), make(12, 8), XDropout(0.3)).to(DEV), make(8, 8).to(DEV)]
    x = torch.randn(size, generator=torch.Generator().manual_seed(1)).to(DEV).requires_grad_()
    a = torch.randn(size, generator=torch.Generator().manual_seed(2)).to(DEV)
    leaves = [x] + [p for part in parts for p in part.parameters()]

    def run(through):
        torch.manual_seed(11)
        for t in leaves:
            t.grad = None
        y = x
        for part in parts:
            y = through(part, y)
        y.backward(a)
        return [y.detach()] + [t.grad for t in leaves]

    want = run(lambda part, y: part(y))
    got = run(lambda part, y: checkpoint(part, y, use_reentrant=reentrant))
    # the same fp32 arithmetic of three layers, whose sums have at most 600 terms; the gradients of other probes differ by their size
    for g, w in zip(got, want):
        assert float((g - w).norm() / w.norm()) <= 4000 * U
