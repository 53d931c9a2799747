"""The optimiser Muon on the device: resuming from a checkpoint."""
import io

import pytest
import torch

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
