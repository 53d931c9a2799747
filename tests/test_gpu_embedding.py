"""Embeddings: the lookup to the last bit, the gradient by sorted indices against sums in 64 bits (token_reference.py)."""
import pytest
import torch

import token_reference as ref
from paper_2106_06998_amd import binding as xb
from paper_2106_06998_amd import embedding as E

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _normal(shape, dtype, seed, scale=1.0):
    return (scale * torch.randn(shape, generator=torch.Generator().manual_seed(seed))).to(dtype).to(DEV)


def _indices(n, rows, kind, seed=5):
    g = torch.Generator().manual_seed(seed)
    if kind == "one":
        return torch.full((n,), rows // 2, dtype=torch.int64, device=DEV)
    if kind == "falling":                    # a few rows make up much of the list
        u = torch.rand(n, generator=g, dtype=torch.float64)
        return ((rows + 1.0) ** u - 1).long().clamp(max=rows - 1).to(DEV)
    if kind == "sorted":
        return torch.randint(rows, (n,), generator=g).sort().values.to(DEV)
    return torch.randint(rows, (n,), generator=g).to(DEV)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n,rows,channels", [(1, 1, 1), (3, 2, 3), (8, 5, 7), (9, 300, 8), (100, 50, 33), (77, 9, 64), (50, 1000, 129), (20, 40, 512), (5, 30, 1000), (8, 100, 4096), (3, 4, 20001)])
def test_lookup(n, rows, channels, dtype):
    w, idx = _normal((rows, channels), TYPES[dtype], 1), _indices(n, rows, "uniform")
    for scale in (1.0, -0.37):
        want = (w.float()[idx] * torch.tensor(scale, dtype=torch.float32)).to(TYPES[dtype])
        assert torch.equal(E.embedding_forward(idx, w, scale), want)
        assert torch.equal(E.embedding_forward(idx.int(), w, scale), want)


GRADIENTS = [(1, 1, 1), (1, 5, 3), (2, 1, 8), (7, 3, 5), (8, 8, 8), (9, 300, 16), (64, 257, 24), (100, 1000, 33), (1000, 7, 40), (1999, 5003, 300), (3000, 70000, 20), (4097, 300, 1000),
             (20000, 1, 17), (30000, 256, 65), (60000, 50000, 24), (65537, 200, 12), (70001, 30000, 33), (300000, 1024, 8), (5000, 300000, 12), (1000, 2000000, 3)]


@pytest.mark.parametrize("kind", ["uniform", "falling", "one", "sorted"])
@pytest.mark.parametrize("n,rows,channels", GRADIENTS)
def test_gradient(n, rows, channels, kind):
    dtype = ("f32", "bf16", "f16")[(n + rows + channels) % 3]
    dy, idx = _normal((n, channels), TYPES[dtype], 2), _indices(n, rows, kind)
    got = E.embedding_backward(dy, idx, rows, 1.7)
    want, off = ref.embedding_gradient(dy, idx, rows, 1.7)
    ref.close(got, want, off)
    assert torch.equal(E.embedding_backward(dy, idx.int(), rows, 1.7), got)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("channels", [1, 2, 3, 4, 7, 8, 9, 15, 16, 31, 64, 65, 250, 256, 257, 511, 512, 513, 1030, 5000])
def test_widths_and_types(channels, dtype):
    dy, idx = _normal((700, channels), TYPES[dtype], 2), _indices(700, 90, "falling")
    want, off = ref.embedding_gradient(dy, idx, 90, 0.5, 3)
    ref.close(E.embedding_backward(dy, idx, 90, 0.5, 3), want, off)
    want, off = ref.embedding_gradient(dy, idx, 90, 0.5, 3, torch.float32)
    got = E.embedding_backward(dy, idx, 90, 0.5, 3, torch.float32)
    assert got.dtype == torch.float32 and bool((got[3] == 0).all())
    ref.close(got, want, off)


@pytest.mark.parametrize("n", [50, 3000, 80000])
def test_indices_outside_the_table(n):
    """rows of NaN in the lookup; no part of the gradient"""
    rows = 40
    idx = _indices(n, rows, "uniform")
    idx[::7] = -1
    idx[3::11] = rows
    idx[5::13] = 2 ** 40
    idx[6::17] = -2 ** 62
    there = (idx >= 0) & (idx < rows)
    w = _normal((rows, 12), torch.float32, 1)
    y = E.embedding_forward(idx, w)
    assert torch.equal(torch.isnan(y).all(1), ~there) and torch.equal(y[there], w[idx[there]])
    dy = _normal((n, 12), torch.float32, 2)
    dy[~there] = float("nan")
    want, off = ref.embedding_gradient(dy, idx, rows, 1.0, 0)
    ref.close(E.embedding_backward(dy, idx, rows, 1.0, 0), want, off)
    nowhere = torch.full((n,), -1, device=DEV)
    assert bool((E.embedding_backward(dy, nowhere, rows) == 0).all())
    assert bool((E.embedding_backward(dy, torch.full((n,), 7, device=DEV), rows, 1.0, 7) == 0).all())


def test_rows_do_not_share_what_is_not_finite():
    dy, idx = _normal((5000, 20), torch.bfloat16, 1), _indices(5000, 100, "falling")
    first = int((idx == 3).nonzero()[0])
    dy[first, 4] = float("nan")
    dy[first, 5] = float("inf")
    got = E.embedding_backward(dy, idx, 100).cpu()
    want = torch.zeros(100, 20, dtype=torch.bool)
    want[3, 4:6] = True
    assert torch.equal(~torch.isfinite(got), want) and bool(torch.isnan(got[3, 4])) and bool(torch.isinf(got[3, 5]))


@pytest.mark.parametrize("n,rows", [(30000, 5000), (200000, 5000), (200000, 300)])
def test_deterministic(n, rows):
    dy, idx = _normal((n, 24), torch.float32, 1), _indices(n, rows, "falling")
    first = E.embedding_backward(dy, idx, rows)
    for _ in range(4):
        assert torch.equal(E.embedding_backward(dy, idx, rows), first)


def test_empty():
    w = _normal((5, 8), torch.float16, 1)
    idx = torch.empty(0, 3, dtype=torch.int64, device=DEV)
    assert E.embedding_forward(idx, w).shape == (0, 3, 8)
    dw = E.embedding_backward(torch.empty(0, 3, 8, dtype=torch.float16, device=DEV), idx, 5)
    assert dw.shape == (5, 8) and bool((dw == 0).all())


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_autograd_and_module(dtype):
    dt = TYPES[dtype]
    m = E.XEmbedding(30, 16, scale=4.0, padding_idx=-1, axis=1, dtype=dt).to(DEV)
    assert bool((m.weight[29] == 0).all()) and m.padding_idx == 29
    idx = _indices(2 * 6 * 5, 30, "uniform").view(2, 6, 5)
    y = m(idx)
    assert y.shape == (2, 16, 6, 5) and y.is_contiguous(memory_format=torch.channels_last)
    assert torch.equal(y.permute(0, 2, 3, 1), E.embedding_forward(idx, m.weight.detach(), 4.0))
    dy = _normal((2, 16, 6, 5), dt, 3)
    y.backward(dy)
    want, off = ref.embedding_gradient(dy.permute(0, 2, 3, 1), idx, 30, 4.0, 29)
    ref.close(m.weight.grad, want, off)
    assert bool((m.weight.grad[29] == 0).all())
    # a broadcast gradient; indices with gaps; a scalar index
    m.weight.grad = None
    gaps = _indices(60, 30, "uniform").view(3, 20)[:, ::3]
    E.embedding(gaps, m.weight, 2.0).sum().backward()
    want, off = ref.embedding_gradient(torch.ones(21, 16, dtype=dt), gaps, 30, 2.0)
    ref.close(m.weight.grad, want, off)
    assert E.embedding(idx[0, 0, 0], m.weight).shape == (16,)
    # a strided table
    wide = _normal((30, 40), dt, 4)
    assert torch.equal(E.embedding_forward(idx, wide[:, 3:20]), E.embedding_forward(idx, wide[:, 3:20].contiguous()))


def test_differences():
    """linear in the table: its difference along v is its value at v"""
    w, v = _normal((50, 24), torch.float32, 1).requires_grad_(), _normal((50, 24), torch.float32, 2)
    a, idx = _normal((400, 24), torch.float32, 3), _indices(400, 50, "falling")
    E.embedding(idx, w, 1.5).backward(a)
    along = float((w.grad.double() * v.double()).sum())
    want = float((v.double()[idx] * 1.5 * a.double()).sum())
    _, off = ref.embedding_gradient(a, idx, 50, 1.5)
    assert abs(along - want) <= float((off * v.cpu().double().abs()).sum()) + 1e-9 * abs(want)


@pytest.mark.parametrize("n,rows", [(500, 60), (90000, 3000)])
def test_streams_and_graphs(n, rows):
    dy, idx, w = _normal((n, 16), torch.bfloat16, 1), _indices(n, rows, "falling"), _normal((rows, 16), torch.bfloat16, 2)
    one = lambda: (E.embedding_forward(idx, w, 2.0), E.embedding_backward(dy, idx, rows, 2.0))
    first = one()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        aside = one()
        beside = one()
    here = one()
    torch.cuda.current_stream().wait_stream(s)
    for got in (aside, beside, here):
        assert all(torch.equal(a, b) for a, b in zip(first, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = one()
    for k in range(4):
        idx.copy_(_indices(n, rows, "uniform" if k % 2 else "falling", k))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        assert all(torch.equal(a, b) for a, b in zip(got, one()))
        torch.cuda.synchronize()


def test_long_runs_and_tables_beyond_32_bits():
    """a table and a gradient of more than 2^32 bytes, the last rows and places named"""
    rows, channels = 2 ** 20 + 3, 2 ** 12
    w = torch.zeros(rows, channels, dtype=torch.bfloat16, device=DEV)
    w[-1] = 3
    idx = torch.tensor([rows - 1, 0, rows - 1], device=DEV)
    y = E.embedding_forward(idx, w, 2.0)
    assert bool((y[0] == 6).all()) and bool((y[1] == 0).all()) and torch.equal(y[0], y[2])
    del w
    dw = E.embedding_backward(torch.ones(3, channels, dtype=torch.bfloat16, device=DEV), idx, rows)
    assert bool((dw[-1] == 2).all()) and bool((dw[0] == 1).all()) and not bool(dw[1:-1].any())
    del dw
    n = 2 ** 19 + 5
    dy = torch.ones(n, 2 ** 13, dtype=torch.bfloat16, device=DEV)
    idx = torch.full((n,), 2, device=DEV)
    idx[-4:] = 1
    dw = E.embedding_backward(dy, idx, 4, dtype=torch.float32)
    assert bool((dw[1] == 4).all()) and bool((dw[2] == n - 4).all()) and not bool(dw[0].any()) and not bool(dw[3].any())


def test_refusals():
    w, idx = torch.ones(6, 4, device=DEV), torch.zeros(3, dtype=torch.int64, device=DEV)
    dy = torch.ones(3, 4, device=DEV)
    for call in (lambda: E.embedding_forward(idx.float(), w), lambda: E.embedding_forward(idx.short(), w), lambda: E.embedding_forward(idx.cpu(), w), lambda: E.embedding_forward(idx, w[0]),
                 lambda: E.embedding_forward(idx, w.double()), lambda: E.embedding_forward(idx, w[:, :0]), lambda: E.embedding_backward(dy[:2], idx, 6), lambda: E.embedding_backward(dy, idx, 0),
                 lambda: E.embedding_backward(dy, idx, 6, 1.0, 6), lambda: E.embedding_backward(dy, idx, 6, dtype=torch.float16), lambda: E.embedding_backward(dy.t(), idx, 6)):
        with pytest.raises(RuntimeError):
            call()
    with pytest.raises(xb.XConvError):
        E.embedding_backward(dy, idx, 2 ** 22 + 1)
    with pytest.raises(xb.XConvError):
        E.embedding_forward(idx, w, float("nan"))
    with pytest.raises(ValueError):
        E.embedding(idx, w, padding_idx=6)
    with pytest.raises(ValueError):
        E.embedding(idx, w, axis=0)
    with pytest.raises(ValueError):
        E.embedding(idx[0], w, axis=1)


def test_places_beyond_32_bits():
    """a table, results, gradients and a gradient's source of more than 2^32 values each; only a few places are not zero"""
    rows, c = 2 ** 31 - 1, 3
    w = torch.zeros(rows, c, dtype=torch.float16, device=DEV)
    w[-4:] = _normal((4, c), torch.float16, 1)
    for idx in (torch.tensor([rows - 1, 0, rows - 4, rows - 2], dtype=t, device=DEV) for t in (torch.int32, torch.int64)):
        assert torch.equal(E.embedding_forward(idx, w), w[idx.long()])
    del w
    n, c = 2 ** 22 + 9, 1032
    w, idx = _normal((50, c), torch.bfloat16, 2), _indices(n, 50, "uniform")
    y = E.embedding_forward(idx, w, 0.5)
    assert torch.equal(y[-20:], w[idx[-20:]] * 0.5) and torch.equal(y[:20], w[idx[:20]] * 0.5)
    y[:-20] = 0
    assert torch.equal(E.embedding_backward(y, idx, 50, 0.25), E.embedding_backward(y[-20:].clone(), idx[-20:].clone(), 50, 0.25))
    del y
    rows = 2 ** 22
    dy, idx = _normal((20000, c), torch.bfloat16, 3), rows - 1 - 7 * _indices(20000, 30, "uniform")
    got = E.embedding_backward(dy, idx, rows, 1.0)
    small, where = E.embedding_backward(dy, (rows - 1 - idx) // 7, 30, 1.0), rows - 1 - 7 * torch.arange(30, device=DEV)
    assert torch.equal(got[where], small)
    got[where] = 0
    assert all(not bool(t.any()) for t in got.split(2 ** 19))


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_widest(dtype):
    """2^24 columns, the most that are taken"""
    c = 2 ** 24
    dy, idx = _normal((20, c), TYPES[dtype], 4), _indices(20, 3, "uniform")
    got = E.embedding_backward(dy, idx, 3, 0.5)
    for at in (0, c // 2 - 3, c - 40):
        part = slice(at, at + 40)
        want, off = ref.embedding_gradient(dy[:, part].contiguous(), idx, 3, 0.5)
        ref.close(got[:, part], want, off)
    assert torch.equal(E.embedding_forward(idx, dy[:3], 2.0), dy[:3][idx] * 2)
