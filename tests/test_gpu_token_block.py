"""Embedding, dropout, norm with residual and convolution together, as a network runs them: against the same network in 64 bits, and
captured into a graph."""
import pytest
import torch

import token_reference as ref
from paper_2106_06998_amd import norm as N
from paper_2106_06998_amd.dropout import XDropout, dropout_forward
from paper_2106_06998_amd.embedding import XEmbedding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _net(dtype, p=0.25):
    torch.manual_seed(3)
    m = torch.nn.ModuleDict({"embed": XEmbedding(40, 32, scale=32 ** 0.5, padding_idx=0), "drop": XDropout(p), "mix": torch.nn.Linear(32, 32),
                             "norm": N.XRMSNorm(32, p=p), "out": N.XRMSNorm(32)})
    return m.to(DEV, dtype)


def _run(m, idx):
    stream = m["drop"](m["embed"](idx))
    y, stream = m["norm"](m["mix"](stream), stream)
    return m["out"](torch.nn.functional.silu(y) + stream)


def test_against_64_bits():
    m = _net(torch.float32)
    idx = torch.randint(0, 40, (6, 21), generator=torch.Generator().manual_seed(1)).to(DEV)
    out = _run(m, idx)
    a = torch.randn(out.shape, generator=torch.Generator().manual_seed(2))
    out.backward(a.to(DEV))
    P = {k: v.detach().cpu().double().requires_grad_() for k, v in m.named_parameters()}
    rms = lambda h, w: h * ((h * h).mean(-1, keepdim=True) + 1e-6) ** -0.5 * w
    x = P["embed.weight"][idx.cpu()] * 32 ** 0.5
    stream = x * ref.mask_like(out, 0.25, m["drop"].last_seed)
    h = stream + (stream @ P["mix.weight"].t() + P["mix.bias"]) * ref.mask_like(out, 0.25, m["norm"].last_seed)
    want = rms(torch.nn.functional.silu(rms(h, P["norm.weight"])) + h, P["out.weight"])
    want.backward(a.double())
    # a chain of some twenty fp32 steps of at most 32 terms: a part in 2^24 of a few hundred
    close = lambda g, w: float((g.detach().cpu().double() - w).norm() / w.norm()) <= 400 * ref.U
    assert close(out, want.detach())
    for k, v in m.named_parameters():
        w = P[k].grad.clone()
        if k == "embed.weight":
            w[0] = 0                        # the padding row learns nothing
        assert close(v.grad, w), k


def test_captured_training_steps():
    """forward, backward and update as one graph whose replays draw their own masks, against eager steps with the same numbers"""
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    idx = torch.randint(0, 40, (6, 21), generator=torch.Generator().manual_seed(1)).to(DEV)
    table = torch.randn(40, 32, generator=torch.Generator().manual_seed(2)).to(DEV)
    w = torch.ones(32, device=DEV)
    r = torch.randn(6, 21, 32, generator=torch.Generator().manual_seed(4)).to(DEV)

    def one(table, w):
        from paper_2106_06998_amd.embedding import embedding_backward, embedding_forward
        x = dropout_forward(embedding_forward(idx, table, 2.0), 0.2, 7, step)
        y, h, rstd = N.rms_norm_forward(x, w, r, 1e-6, -1, 0.3, 8, step)
        dx, _, dw = N.rms_norm_backward(y - r, h, rstd, w, h, -1, 0.3, 8, step)
        dt = embedding_backward(dropout_forward(dx, 0.2, 7, step), idx, 40, 2.0, 0)
        table.sub_(dt, alpha=0.01)
        w.sub_(dw, alpha=0.001)
        step.add_(1)

    t0, w0 = table.clone(), w.clone()
    one(t0, w0)                             # everything has run once
    t0, w0 = table.clone(), w.clone()
    step.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one(table, w)
    step.zero_()
    for k in range(5):
        graph.replay()
        torch.cuda.synchronize()
        step.sub_(1)
        one(t0, w0)
        torch.cuda.synchronize()
        assert torch.equal(table, t0) and torch.equal(w, w0) and int(step) == k + 1
    assert bool(torch.isfinite(table).all())
