"""The optimiser Muon on the device: resuming from a checkpoint."""
import io

import pytest
import torch

from paper_2106_06998_amd import binding as xb
from paper_2106_06998_amd import optim
from test_gpu_orth import DEV, TD, gradient, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_a_resumed_run_goes_on_with_the_same_bits(dtype):
    say("Muon, resumed", dtype)
    shapes = [(24, 40), (100, 90), (16, 9, 3, 3)]
    grads = [[gradient(s[0], torch.Size(s[1:]).numel(), 10 * t + i, dtype).view(s).to(DEV) for i, s in enumerate(shapes)] for t in range(4)]

    def fresh():
        return [torch.nn.Parameter((0.1 * gradient(s[0], torch.Size(s[1:]).numel(), 50 + i, scale=1.0)).view(s).to(TD[dtype]).to(DEV)) for i, s in enumerate(shapes)]

    def steps(params, opt, which):
        for t in which:
            for p, g in zip(params, grads[t]):
                p.grad = g.clone()
            opt.step()

    whole = fresh()
    steps(whole, optim.Muon(whole, lr=0.05, momentum=0.9), range(4))
    half = fresh()
    opt = optim.Muon(half, lr=0.05, momentum=0.9)
    steps(half, opt, range(2))
    file = io.BytesIO()
    torch.save({"weights": [p.detach() for p in half], "optimiser": opt.state_dict()}, file)
    file.seek(0)
    saved = torch.load(file, weights_only=True, map_location="cpu")
    rest = [torch.nn.Parameter(w.to(DEV)) for w in saved["weights"]]
    new = optim.Muon(rest, lr=0.5)
    new.load_state_dict(saved["optimiser"])
    steps(rest, new, range(2, 4))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(whole, rest))


def some(rows, cols, dtype, seed=1):
    """A weight, a gradient and a momentum, and copies of the first and the last."""
    w, g = (gradient(rows, cols, seed + i, dtype).to(DEV) for i in range(2))
    m = gradient(rows, cols, seed + 2).to(DEV)
    return (w, g, m), (w.clone(), m.clone())


def untouched(tensors, copies, versions):
    torch.cuda.synchronize()
    (w, _, m), (w0, m0) = tensors, copies
    return torch.equal(w, w0) and torch.equal(m, m0) and (w._version, m._version) == versions


def test_a_refused_step_changes_nothing():
    """Weights of two types are two calls of the library: when the second one's shape is refused, the first one has not run."""
    small, copies = some(40, 60, "f32")
    versions = (small[0]._version, small[2]._version)
    n = (1 << 24) + 1
    far = [torch.zeros(1, n, dtype=torch.float16, device=DEV) for _ in range(2)] + [torch.zeros(1, n, device=DEV)]
    with pytest.raises(xb.XConvError):
        optim.muon_step([small[0]], [small[1]], [small[2]], float("inf"))
    assert untouched(small, copies, versions)
    say("muon_step, f32 40 x 60 and a refused f16 1 x %d" % n)
    with pytest.raises(xb.XConvError, match="unsupported"):
        optim.muon_step([small[0], far[0]], [small[1], far[1]], [small[2], far[2]], 0.1)
    assert untouched(small, copies, versions)


def test_a_step_without_room_for_its_scratch_changes_nothing():
    small, copies = some(40, 60, "f32")
    versions = (small[0]._version, small[2]._version)
    large = [torch.zeros(2048, 4096, dtype=torch.float16, device=DEV) for _ in range(2)] + [torch.zeros(2048, 4096, device=DEV)]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    say("muon_step, f32 40 x 60 and f16 2048 x 4096 without room for its scratch")
    total = torch.cuda.get_device_properties(0).total_memory
    try:
        # (the scratch of 2048 x 4096 takes over 100 MB)
        torch.cuda.set_per_process_memory_fraction((torch.cuda.memory_reserved() + (32 << 20)) / total)
        with pytest.raises(torch.OutOfMemoryError):
            optim.muon_step([small[0], large[0]], [small[1], large[1]], [small[2], large[2]], 0.1)
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    assert untouched(small, copies, versions)
    optim.muon_step([small[0], large[0]], [small[1], large[1]], [small[2], large[2]], 0.1)
    torch.cuda.synchronize()
    assert small[0]._version > versions[0] and small[2]._version > versions[1] and not torch.equal(small[0], copies[0])


def test_a_graph_knows_that_a_strided_weight_has_changed():
    """Weights and momenta whose memory has gaps are updated through a copy: their versions count as well."""
    big = torch.randn(12, 40, device=DEV)
    w = big[:, ::2].requires_grad_(True)
    m = torch.zeros(12, 40, device=DEV)[:, ::2]
    y = (w * w).sum()
    before, before_m = w._version, m._version
    optim.muon_step([w.detach()], [torch.ones(12, 20, device=DEV)], [m], 0.1)
    torch.cuda.synchronize()
    assert w._version > before and m._version > before_m and bool(m.any())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_an_expanded_momentum_or_weight_is_refused_before_anything_runs():
    small, copies = some(40, 60, "f32")
    versions = (small[0]._version, small[2]._version)
    w, g, m = (torch.zeros(12, 20, device=DEV) for _ in range(3))
    one = torch.zeros(1, 20, device=DEV).expand(12, 20)
    for bad in ((w, g, one), (one, g, m)):
        with pytest.raises(RuntimeError, match="single memory location"):
            optim.muon_step([small[0], bad[0]], [small[1], bad[1]], [small[2], bad[2]], 0.1)
        assert untouched(small, copies, versions)
    optim.muon_step([w], [torch.ones(1, 20, device=DEV).expand(12, 20)], [m], 0.1)        # (a gradient may be)
    assert bool(w.any())


def test_tensors_over_each_other_are_refused():
    """The same weight twice, a momentum over another one's end, a momentum that is a gradient: two workgroups would race."""
    (w, g, m), copies = some(40, 60, "f32")
    versions = (w._version, m._version)
    other, buf = torch.zeros(40, 60, device=DEV), torch.zeros(41, 60, device=DEV)
    gaps = torch.zeros(40, 120, device=DEV)[:, ::2]
    for call in (([w, w], [g, g], [m, other]), ([w, other], [g, g], [m, m]), ([w, other], [g, g], [buf[:40], buf[1:]]), ([w], [g], [g]),
                 ([w, other], [g, m], [m, buf[1:]]), ([gaps, gaps], [g, g], [m, other])):
        with pytest.raises(RuntimeError, match="lies over another tensor"):
            optim.muon_step(*call, 0.1)
    assert untouched((w, g, m), copies, versions) and not other.any() and not buf.any()
    # neighbours in one buffer, one gradient for two weights and columns between each other are fine
    pair = torch.zeros(2, 40, 60, device=DEV)
    optim.muon_step([pair[0], pair[1]], [g, g], [m, other], 0.1)
    cols = torch.zeros(40, 120, device=DEV)
    optim.muon_step([cols[:, ::2], cols[:, 1::2]], [g, g], [buf[1:], torch.zeros(40, 60, device=DEV)], 0.1)
    torch.cuda.synchronize()
    assert bool(pair[0].any()) and bool(pair[1].any()) and torch.equal(cols[:, ::2], cols[:, 1::2])
