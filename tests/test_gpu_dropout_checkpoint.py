"""Gradients under activation checkpointing: the parts that are run again for the backward pass apply the masks that the loss saw."""
import pytest
import torch
from torch.utils.checkpoint import checkpoint

import token_reference as ref
from paper_2106_06998_amd.dropout import XDropout
from paper_2106_06998_amd.layer import convert_net
from paper_2106_06998_amd.norm import XRMSNorm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class _Branch(torch.nn.Module):
    def __init__(self):
        super().__init__()
        self.mix, self.norm = torch.nn.Linear(32, 32), XRMSNorm(32, p=0.4)

    def forward(self, x):
        y, h = self.norm(self.mix(x), x)
        return y + h


def _dropped():
    return torch.nn.Sequential(torch.nn.Linear(32, 32), XDropout(0.5), torch.nn.Linear(32, 32))


def _converted():
    net = torch.nn.Sequential(torch.nn.Linear(32, 32), torch.nn.Dropout(0.5), torch.nn.Linear(32, 32), torch.nn.Dropout(0.2))
    convert_net(net, dropout=True)
    assert type(net[1]) is type(net[3]) is XDropout
    return net


@pytest.mark.parametrize("reentrant", [False, True])
@pytest.mark.parametrize("make", [_dropped, _Branch, _converted], ids=["dropout", "norm", "converted"])
def test_gradients(make, reentrant):
    torch.manual_seed(3)
    parts = [make().to(DEV) for _ in range(2)]
    x = torch.randn(50, 32, generator=torch.Generator().manual_seed(1)).to(DEV).requires_grad_()
    a = torch.randn(50, 32, generator=torch.Generator().manual_seed(2)).to(DEV)
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
    # the same fp32 arithmetic; a product may take its sums of 32 or 50 terms in another order in each of some ten layers
    for g, w in zip(got, want):
        assert float((g - w).norm() / w.norm()) <= 500 * ref.U
