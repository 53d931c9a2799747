"""Host side of dropout, the root-mean-square norm and embeddings: structures, sizes, statuses, masks and refusals, without a GPU."""
import ctypes

import numpy as np
import pytest
import torch

import token_reference as ref
from paper_2106_06998_amd import binding as xb
from paper_2106_06998_amd import dropout, embedding, norm

A, B, C, D, E, F = (ctypes.c_void_p(1 << k) for k in range(40, 46))         # never dereferenced: validation fails first
ODD = ctypes.c_void_p((1 << 40) + 1)


def test_structures_match_the_header():
    assert ctypes.sizeof(xb.xconv_drop) == 24 and xb.xconv_drop.step_dev.offset == 8 and xb.xconv_drop.drop_q16.offset == 16
    assert ctypes.sizeof(xb.xconv_embed_desc) == 40 and xb.xconv_embed_desc.C.offset == 16 and xb.xconv_embed_desc.scale.offset == 32


@pytest.mark.parametrize("seed", [0, 5, 2 ** 64 - 1])
@pytest.mark.parametrize("q", [0, 1, 6554, 32768, 65535, 65536])
def test_masks(seed, q):
    for first in (0, 3, 2 ** 33 + 5):
        got = xb.xconv_dropout_mask(xb.make_drop(seed, q), first, 50)
        assert got.tolist() == [ref.kept_one(seed, q, first + i) for i in range(50)] == ref.kept(seed, q, first, 50).tolist()
    many = ref.kept(seed, q, 0, 1 << 16)
    share = 1 - q / 65536
    assert abs(many.mean() - share) <= 6 * (share * (1 - share) / (1 << 16)) ** 0.5        # six deviations


def test_masks_of_seeds_and_lanes_are_unlike():
    """no two of eight seeds and four fields agree on more than fair coins do"""
    m = np.stack([ref.kept(s, 32768, 0, 1 << 14) for s in range(8)])
    rows = np.concatenate([m.reshape(8, -1, 4).transpose(0, 2, 1).reshape(32, -1)])
    agree = (2.0 * rows - 1) @ (2.0 * rows - 1).T / rows.shape[1]
    assert np.abs(agree - np.eye(32)).max() <= 6 / rows.shape[1] ** 0.5


def test_dropout_statuses():
    L = xb.lib()
    good = xb.make_drop(1, 100)
    run = lambda drop=good, dtype=0, x=A, y=B, n=4: L.xconv_dropout(dtype, x, y, n, ctypes.byref(drop) if drop is not None else None, None)
    assert run(n=0) == xb.XCONV_OK and run(n=0, x=None, y=None) == xb.XCONV_OK
    assert run(n=-1) == run(dtype=3) == run(dtype=-1) == run(x=None) == run(y=None) == run(drop=None) == run(x=ODD) == run(y=ODD) == xb.XCONV_EINVAL
    assert run(drop=xb.make_drop(1, -1)) == run(drop=xb.make_drop(1, 65537)) == xb.XCONV_EINVAL
    assert run(drop=xb.xconv_drop(1, 4097, 100)) == xb.XCONV_EINVAL
    assert run(n=(1 << 40) + 1) == xb.XCONV_EUNSUPPORTED
    assert run(y=ctypes.c_void_p((1 << 40) + 4)) == xb.XCONV_EINVAL         # over a part of its input
    assert run(drop=xb.xconv_drop(1, (1 << 41) + 8, 100)) == xb.XCONV_EINVAL   # over the step
    mask = (ctypes.c_uint8 * 4)()
    call = lambda d, first, n, p: L.xconv_dropout_mask(ctypes.byref(d) if d is not None else None, first, n, p)
    assert call(None, 0, 4, mask) == call(good, -1, 4, mask) == call(good, 0, -1, mask) == call(good, 0, 4, None) == call(xb.xconv_drop(1, 4096, 100), 0, 4, mask) == xb.XCONV_EINVAL
    assert call(good, 0, 0, None) == xb.XCONV_OK


def test_rms_statuses():
    L = xb.lib()
    good = lambda: xb.make_norm_desc(10, 24, 6, "bf16", "f32")
    fwd = lambda d, x=A, r=B, g=C, y=D, h=E, s=F, drop=None: L.xconv_rmsnorm_fwd(ctypes.byref(d) if d is not None else None, x, r, g, y, h, s, drop, None)
    fwd8 = lambda d, x=A, r=B, g=C, q=D, s=F, h=E, t=0: L.xconv_rmsnorm_fwd_8bit(ctypes.byref(d), t, x, r, g, q, s, h, None)
    W = ctypes.c_void_p(1 << 46)
    bwd = lambda d, dy=A, h=B, s=F, g=C, dh=D, dx=E, dr=ctypes.c_void_p(1 << 39), dw=ctypes.c_void_p(1 << 38), ws=W, n=1 << 30, drop=None: L.xconv_rmsnorm_bwd(
        ctypes.byref(d), dy, h, s, g, dh, dx, dr, dw, ws, n, drop, None)
    assert fwd(None) == xb.XCONV_EINVAL
    for field, value, status in (("outer", -1, 1), ("inner", 0, 1), ("C", 0, 1), ("dtype", 3, 1), ("w_dtype", xb.XCONV_F16, 1), ("eps", -1.0, 1), ("eps", float("nan"), 1),
                                 ("C", (1 << 24) + 1, 2), ("inner", (1 << 30) + 1, 2), ("outer", 1 << 40, 2)):
        d = good()
        setattr(d, field, value)
        assert fwd(d) == fwd8(d) == bwd(d) == status, field
        assert xb.xconv_rmsnorm_workspace_bytes(d) == 0
    huge = xb.make_norm_desc(1 << 39, 1 << 10)
    assert fwd(huge) == bwd(huge) == xb.XCONV_EUNSUPPORTED
    d = good()
    for bad in (dict(x=None), dict(y=None), dict(x=ODD), dict(r=ODD), dict(y=ODD), dict(h=ODD), dict(g=ctypes.c_void_p((1 << 42) + 2)), dict(s=ctypes.c_void_p((1 << 45) + 2)),
                dict(y=E), dict(y=ctypes.c_void_p((1 << 40) + 2)), dict(h=ctypes.c_void_p((1 << 41) + 2)), dict(s=D), dict(s=A), dict(g=E),
                dict(drop=ctypes.byref(xb.make_drop(0, 65537))), dict(drop=ctypes.byref(xb.xconv_drop(0, 4100, 5)))):
        assert fwd(d, **bad) == xb.XCONV_EINVAL, bad
    for bad in (dict(x=None), dict(q=None), dict(s=None), dict(t=2), dict(t=-1), dict(q=A), dict(q=B), dict(q=E), dict(h=F), dict(s=D), dict(h=ODD)):
        assert fwd8(d, **bad) == xb.XCONV_EINVAL, bad
    for bad in (dict(dy=None), dict(h=None), dict(s=None), dict(ws=None), dict(dx=ODD), dict(dh=ODD), dict(dr=E), dict(dw=C), dict(ws=A), dict(dw=W), dict(dx=ctypes.c_void_p((1 << 40) + 2)),
                dict(ws=ctypes.c_void_p((1 << 46) + 2)), dict(drop=ctypes.byref(xb.make_drop(0, -1)))):
        assert bwd(d, **bad) == xb.XCONV_EINVAL, bad
    assert xb.xconv_rmsnorm_workspace_bytes(d) >= 24 * 4
    assert bwd(d, n=16) == xb.XCONV_EWORKSPACE
    assert bwd(d, dx=None, dr=None, dw=None, dy=None) == xb.XCONV_OK         # nothing is wanted
    empty = xb.make_norm_desc(0, 24)
    assert fwd(empty, x=None, y=None) == fwd8(empty, x=None, q=None, s=None) == bwd(empty, dw=None) == xb.XCONV_OK


def test_embedding_statuses():
    L = xb.lib()
    good = lambda **kw: xb.make_embed_desc(**{**dict(n=10, rows=5, C=8, dtype="bf16"), **kw})
    fwd = lambda d, i=A, w=B, y=C: L.xconv_embed_fwd(ctypes.byref(d) if d is not None else None, i, w, y, None)
    bwd = lambda d, i=A, dy=B, dw=C, t=1, ws=D, n=1 << 40: L.xconv_embed_bwd(ctypes.byref(d) if d is not None else None, i, dy, dw, t, ws, n, None)
    assert fwd(None) == bwd(None) == xb.XCONV_EINVAL
    for kw, status in ((dict(n=-1), 1), (dict(rows=0), 1), (dict(C=0), 1), (dict(dtype=3), 1), (dict(scale=float("inf")), 1), (dict(scale=float("nan")), 1), (dict(padding_idx=5), 1),
                       (dict(padding_idx=-2), 1), (dict(n=(1 << 27) + 1), 2), (dict(C=(1 << 24) + 1), 2), (dict(rows=1 << 31), 2)):
        assert fwd(good(**kw)) == bwd(good(**kw)) == status, kw
        assert xb.xconv_embed_workspace_bytes(good(**kw)) == 0
    assert bwd(good(rows=(1 << 22) + 1)) == xb.XCONV_EUNSUPPORTED
    d = good()
    for bad in (dict(i=None), dict(w=None), dict(y=None), dict(i=ctypes.c_void_p((1 << 40) + 4)), dict(w=ODD), dict(y=ODD), dict(y=B), dict(y=A)):
        assert fwd(d, **bad) == xb.XCONV_EINVAL, bad
    for bad in (dict(i=None), dict(dy=None), dict(dw=None), dict(ws=None), dict(t=2), dict(t=3), dict(ws=ctypes.c_void_p((1 << 43) + 16)), dict(dw=B), dict(ws=B), dict(dw=D), dict(dy=ODD)):
        assert bwd(d, **bad) == xb.XCONV_EINVAL, bad
    assert bwd(d, n=64) == xb.XCONV_EWORKSPACE
    assert fwd(good(n=0), i=None, w=None, y=None) == xb.XCONV_OK
    # the scratch grows with the list, not with the product of list and table
    small, large = xb.xconv_embed_workspace_bytes(good(n=1 << 20)), xb.xconv_embed_workspace_bytes(good(n=1 << 20, rows=1 << 20))
    assert 0 < small < large <= small + 16 * (1 << 20) + (4 << 20)


def test_python_refusals_without_a_gpu():
    x, i = torch.zeros(3, 4), torch.zeros(3, dtype=torch.int64)
    for call in (lambda: dropout.dropout_forward(x, 0.5, 1), lambda: dropout.dropout_backward(x, 0.5, 1), lambda: dropout.dropout(x, 0.5, 1), lambda: norm.rms_norm_forward(x),
                 lambda: norm.rms_norm_backward(x, x, x), lambda: norm.rms_norm(x), lambda: norm.rms_norm_8bit(x), lambda: embedding.embedding_forward(i, x),
                 lambda: embedding.embedding_backward(x, i, 5), lambda: embedding.embedding(i, x), lambda: dropout.XDropout()(x), lambda: embedding.XEmbedding(5, 4)(i)):
        with pytest.raises(RuntimeError, match="GPU only"):
            call()
    for make in (lambda: dropout.XDropout(-0.1), lambda: dropout.XDropout(1.1), lambda: dropout.XDropout(float("nan")), lambda: norm.XRMSNorm(0), lambda: norm.XRMSNorm(4, axis=2),
                 lambda: norm.XRMSNorm(4, eps=-1.0), lambda: norm.XRMSNorm(4, p=2.0), lambda: embedding.XEmbedding(0, 4), lambda: embedding.XEmbedding(4, 0),
                 lambda: embedding.XEmbedding(4, 4, padding_idx=4), lambda: embedding.XEmbedding(4, 4, axis=2), lambda: embedding.XEmbedding(4, 4, scale=float("inf"))):
        with pytest.raises(ValueError):
            make()
    assert dropout.XDropout().eval()(x) is x
    assert "p=0.5" in repr(dropout.XDropout()) and "axis=1" in repr(norm.XRMSNorm(4, axis=1)) and "5, 4" in repr(embedding.XEmbedding(5, 4))
