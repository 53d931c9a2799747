"""The example on maps of codes: it runs in every storage type, and the gradients of its embedding, norms and head are those of the same
network in 64 bits (the convolutions' own are estimates)."""
import math

import pytest
import torch
import torch.nn.functional as F

import token_reference as ref
from paper_2106_06998_amd import train_example as ex

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_it_runs(dtype):
    losses, wrong = ex.train(6, dtype, batch_size=16, report=lambda *a: None, codes=True)
    assert len(losses) == 6 and all(math.isfinite(v) for v in losses) and 0 <= wrong <= 1


def test_gradients():
    torch.manual_seed(2)
    net = ex.CodeNet(width=32, r=8, blocks=2, p=0.25).cuda()
    codes = torch.randint(0, ex.CODES, (3, 8, 8), generator=torch.Generator().manual_seed(1))
    out = net(codes.cuda())
    a = torch.randn(out.shape, generator=torch.Generator().manual_seed(2))
    out.backward(a.cuda())
    P = {k: v.detach().cpu().double().requires_grad_() for k, v in net.named_parameters()}

    def mask(seed):
        # channels-last activations: places in that order
        like = torch.empty(3, 32, 8, 8).contiguous(memory_format=torch.channels_last)
        return ref.mask_like(like, 0.25, seed)

    rms = lambda h, w: h * ((h * h).mean(1, keepdim=True) + 1e-6) ** -0.5 * w.view(1, -1, 1, 1)
    stream = P["embed.weight"][codes].permute(0, 3, 1, 2) * mask(net.drop.last_seed)
    y = rms(stream, P["norm.weight"])
    for i, b in enumerate(net.blocks):
        stream = stream + F.relu(F.conv2d(y, P["blocks.%d.conv.weight" % i], padding=1)) * mask(b.norm.last_seed)
        y = rms(stream, P["blocks.%d.norm.weight" % i])
    want = F.linear(y.mean((2, 3)), P["head.weight"], P["head.bias"])
    want.backward(a.double())
    # a chain of some thirty fp32 steps, sums of up to 288 terms among them
    close = lambda g, w: float((g.detach().cpu().double() - w).norm() / w.norm()) <= 2000 * ref.U
    assert close(out, want.detach())
    for k, v in net.named_parameters():
        assert v.grad is not None and bool(torch.isfinite(v.grad).all()), k
        if "conv" not in k:
            assert close(v.grad, P[k].grad), k
