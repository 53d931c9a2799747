"""Dropout without a stored mask against masks drawn with Python's integers, to the last bit: products are fp32 products, rounded once."""
import numpy as np
import pytest
import torch

import token_reference as ref
from paper_2106_06998_amd import binding as xb
from paper_2106_06998_amd import dropout as D
from paper_2106_06998_amd.layer import convert_net

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _normal(shape, dtype, seed=1):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def _want(x, p, seed, step=0):
    """x: on the CPU"""
    keep = ref.mask_like(x, p, seed, step) != 0
    return torch.where(keep, x.float() * np.float32(ref.factor(p)), torch.zeros((), dtype=torch.float32)).to(x.dtype)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 7, 8, 9, 63, 64, 257, 2047, 2048, 100003])
def test_sizes(n, dtype):
    x = _normal((n,), TYPES[dtype])
    y = D.dropout_forward(x.to(DEV), 0.3, 77)
    assert torch.equal(y.cpu(), _want(x, 0.3, 77))
    assert torch.equal(D.dropout_backward(x.to(DEV), 0.3, 77).cpu(), y.cpu())


@pytest.mark.parametrize("p", [0.0, 1e-6, 2.0 ** -16, 0.1, 0.5, 0.9, 1 - 2.0 ** -16, 1 - 1e-6, 1.0])
def test_rates(p):
    x = _normal((4099,), torch.float32)
    y = D.dropout_forward(x.to(DEV), p, 3).cpu()
    assert torch.equal(y, _want(x, p, 3))
    q = ref.q16(p)
    dropped = int((y == 0).sum())
    # of 4099 independent fair draws: within six deviations
    assert abs(dropped - 4099 * q / 65536) <= 6 * (4099 * q / 65536 * (1 - q / 65536)) ** 0.5 + 1e-9


@pytest.mark.parametrize("seed", [0, 1, -1, 2 ** 63 - 1, 2 ** 63, 2 ** 64 - 1, 2 ** 70 + 5])
def test_any_seed(seed):
    x = _normal((333,), torch.float32)
    assert torch.equal(D.dropout_forward(x.to(DEV), 0.25, seed).cpu(), _want(x, 0.25, seed & (2 ** 64 - 1)))


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("layout", ["planes", "channels_last", "volume", "permuted", "sliced", "expanded", "offset", "empty", "scalar"])
def test_layouts(layout, dtype):
    dt = TYPES[dtype]
    x = {
        "planes": lambda: _normal((3, 5, 7, 9), dt),
        "channels_last": lambda: _normal((3, 5, 7, 9), dt).contiguous(memory_format=torch.channels_last),
        "volume": lambda: _normal((2, 3, 4, 5, 6), dt).contiguous(memory_format=torch.channels_last_3d),
        "permuted": lambda: _normal((6, 10, 11), dt).permute(2, 0, 1),
        "sliced": lambda: _normal((9, 20), dt)[:, 3:17],
        "expanded": lambda: _normal((1, 21), dt).expand(5, 21),
        "offset": lambda: _normal((103,), dt)[1:],
        "empty": lambda: _normal((0, 4), dt),
        "scalar": lambda: _normal((), dt),
    }[layout]()
    dense = x if layout not in ("sliced", "expanded") else x.contiguous()
    g = x.to(DEV) if layout not in ("sliced", "expanded", "offset", "permuted") else None
    if layout == "sliced":
        g = _normal((9, 20), dt).to(DEV)[:, 3:17]
    elif layout == "expanded":
        g = _normal((1, 21), dt).to(DEV).expand(5, 21)
    elif layout == "offset":
        g = _normal((103,), dt).to(DEV)[1:]
    elif layout == "permuted":
        g = _normal((6, 10, 11), dt).to(DEV).permute(2, 0, 1)
    y = D.dropout_forward(g, 0.4, 9)
    assert torch.equal(y.cpu(), _want(dense, 0.4, 9)) and y.shape == x.shape


def test_dropped_places_hide_infinities_and_nan():
    x = torch.full((64,), float("nan"))
    x[::2] = float("inf")
    y = D.dropout_forward(x.to(DEV), 0.5, 4).cpu()
    keep = torch.from_numpy(ref.kept(4, 32768, 0, 64))
    assert 0 < int(keep.sum()) < 64
    assert bool((y[~keep] == 0).all()) and torch.equal(torch.isnan(y), keep & torch.isnan(x)) and torch.equal(torch.isinf(y), keep & torch.isinf(x))
    assert bool((D.dropout_forward(x.to(DEV), 1.0, 4) == 0).all())


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_gradient_uses_the_mask_of_the_forward_pass(dtype):
    dt = TYPES[dtype]
    for fmt in (torch.contiguous_format, torch.channels_last):
        x = _normal((2, 6, 5, 3), dt).contiguous(memory_format=fmt).to(DEV).requires_grad_()
        y = D.dropout(x, 0.3, 5)
        dy = _normal((2, 6, 5, 3), dt, 2).to(DEV)          # (planes, whatever x is)
        y.backward(dy)
        want = _want(dy.cpu().contiguous(memory_format=fmt), 0.3, 5)
        assert torch.equal(x.grad.cpu(), want)
    # a broadcast gradient, and one of another type
    x = _normal((40,), dt).to(DEV).requires_grad_()
    D.dropout(x, 0.3, 5).sum().backward()
    assert torch.equal(x.grad.cpu(), _want(torch.ones(40, dtype=dt), 0.3, 5))


def test_differences():
    """the function is linear: its difference along v is its value at v"""
    x, v = _normal((1001,), torch.float32).to(DEV).requires_grad_(), _normal((1001,), torch.float32, 2).to(DEV)
    w = _normal((1001,), torch.float32, 3).to(DEV)
    D.dropout(x, 0.3, 5).backward(w)
    along = float((x.grad.double() * v.double()).sum())
    want = float((D.dropout_forward(v, 0.3, 5).double() * w.double()).sum())
    size = float((v.double() * w.double()).abs().sum()) * ref.factor(0.3)
    assert abs(along - want) <= 4 * ref.U * size


def test_step_is_added_to_the_seed():
    x = _normal((500,), torch.float32)
    for step in (0, 3, -2, 2 ** 62):
        t = torch.tensor([step], device=DEV)
        assert torch.equal(D.dropout_forward(x.to(DEV), 0.4, 11, t).cpu(), _want(x, 0.4, 11, step))
    t = torch.tensor(1, device=DEV)
    xg = x.to(DEV).requires_grad_()
    y = D.dropout(xg, 0.4, 11, t)
    t += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_a_captured_graph_draws_other_masks():
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    x, dy = _normal((3000,), torch.float16).to(DEV), _normal((3000,), torch.float16, 2).to(DEV)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    D.dropout_forward(x, 0.3, 8, step)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y.copy_(D.dropout_forward(x, 0.3, 8, step))
        dx.copy_(D.dropout_backward(dy, 0.3, 8, step))
        step += 1
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y.cpu(), _want(x.cpu(), 0.3, 8, k)) and torch.equal(dx.cpu(), _want(dy.cpu(), 0.3, 8, k))
        D.dropout_forward(dy, 0.5, k)
        torch.cuda.synchronize()


def test_module_in_a_capture_wants_a_step():
    x = torch.ones(64, device=DEV)
    m = D.XDropout(0.5)
    m(x)
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="captured graph"):
        with torch.cuda.graph(graph):
            m(x)
    torch.cuda.synchronize()
    m.step = torch.zeros(1, dtype=torch.int64, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = m(x)
    for k in range(3):
        m.step.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y.cpu(), _want(x.cpu(), 0.5, m.last_seed, k))


def test_module():
    m = D.XDropout(0.25)
    x = _normal((64, 33), torch.bfloat16).to(DEV).requires_grad_()
    y = m(x)
    assert torch.equal(y.detach().cpu(), _want(x.detach().cpu(), 0.25, m.last_seed))
    first = m.last_seed
    y2 = m(x)
    assert m.last_seed != first and not torch.equal(y, y2)
    y.sum().backward()                                     # the mask of its own forward pass, not of the latest
    assert torch.equal(x.grad.cpu(), _want(torch.ones_like(x).cpu(), 0.25, first))
    assert m.eval()(x) is x and D.XDropout(0.0)(x) is x


def test_conversion_of_a_network():
    net = torch.nn.Sequential(torch.nn.Conv2d(3, 4, 3), torch.nn.Dropout(0.3), torch.nn.Sequential(torch.nn.Dropout(0.1, inplace=True))).to(DEV)
    same, n = convert_net(net, r=2, dropout=True)
    assert same is net and n == 1 and type(net[1]) is D.XDropout and net[1].p == 0.3 and type(net[2][0]) is D.XDropout
    net(torch.ones(2, 3, 8, 8, device=DEV)).sum().backward()
    plain = torch.nn.Sequential(torch.nn.Dropout(0.3))
    convert_net(plain)
    assert type(plain[0]) is torch.nn.Dropout


def test_other_streams_and_in_place():
    x = _normal((200000,), torch.float16)
    g = x.to(DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y = D.dropout_forward(g, 0.3, 5)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y.cpu(), _want(x, 0.3, 5))
    xb.xconv_dropout("f16", g, g, g.numel(), xb.make_drop(5, ref.q16(0.3)))
    torch.cuda.synchronize()
    assert torch.equal(g, y)


def test_places_beyond_32_bits():
    """2^32 + 21 values: the places that the last ones count from pass 32 bits"""
    n = 2 ** 32 + 21
    x = torch.ones(n, dtype=torch.bfloat16, device=DEV)
    y = D.dropout_forward(x, 0.5, 6)
    del x
    for first in (0, 2 ** 31 - 8, 2 ** 32 - 8, n - 40):
        want = torch.from_numpy(ref.kept(6, 32768, first, 40)).to(torch.bfloat16) * 2
        assert torch.equal(y[first:first + 40].cpu(), want[:min(40, n - first)])


def test_refusals():
    x = torch.ones(8, device=DEV)
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(ValueError):
            D.dropout_forward(x, p, 0)
    for step in (torch.zeros(1, device=DEV), torch.zeros(2, dtype=torch.int64, device=DEV), torch.zeros(1, dtype=torch.int64)):
        with pytest.raises(RuntimeError, match="step"):
            D.dropout_forward(x, 0.5, 0, step)
    with pytest.raises(RuntimeError, match="storage type"):
        D.dropout_forward(x.double(), 0.5, 0)
    with pytest.raises(xb.XConvError):
        xb.xconv_dropout("f32", x[:4], x[1:5], 4, xb.make_drop(0, 100))
