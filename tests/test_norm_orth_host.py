"""Host side of the layer normalisation and of the orthogonalised updates: structures, sizes, statuses and refusals, without a GPU."""
import ctypes

import pytest
import torch

from paper_2106_06998_amd import binding as xb
from paper_2106_06998_amd import norm, optim

ONE = ctypes.c_void_p(4096)          # never dereferenced: validation fails first


def test_structures_match_the_header():
    assert ctypes.sizeof(xb.xconv_norm_desc) == 32 and xb.xconv_norm_desc.C.offset == 16
    assert ctypes.sizeof(xb.xconv_orth_item) == 32 and xb.xconv_orth_item.G_dev.offset == 8
    assert ctypes.sizeof(xb.xconv_orth_args) == 28 and ctypes.sizeof(xb.xconv_muon_args) == 16


def test_norm_statuses():
    L = xb.lib()
    good = lambda: xb.make_norm_desc(10, 24, 6, "bf16", "f32")
    assert xb.xconv_layernorm_workspace_bytes(good()) >= 2 * 24 * 4
    assert L.xconv_layernorm_fwd(None, ONE, None, None, ONE, None, None, None) == xb.XCONV_EINVAL
    for field, value, status in (("outer", -1, 1), ("inner", 0, 1), ("C", 0, 1), ("dtype", 3, 1), ("w_dtype", xb.XCONV_F16, 1), ("eps", -1.0, 1), ("eps", float("nan"), 1),
                                 ("eps", float("inf"), 1), ("C", (1 << 24) + 1, 2), ("inner", (1 << 30) + 1, 2), ("outer", 1 << 40, 2)):
        d = good()
        setattr(d, field, value)
        assert L.xconv_layernorm_fwd(ctypes.byref(d), ONE, None, None, ONE, None, None, None) == status, field
        assert L.xconv_layernorm_bwd(ctypes.byref(d), ONE, ONE, ONE, ONE, None, ONE, ONE, ONE, ONE, 1 << 30, None) == status, field
        assert xb.xconv_layernorm_workspace_bytes(d) == 0
    p = ctypes.byref(good())
    odd = ctypes.c_void_p(4097)
    assert L.xconv_layernorm_fwd(p, None, None, None, ONE, None, None, None) == xb.XCONV_EINVAL
    assert L.xconv_layernorm_fwd(p, ONE, None, None, None, None, None, None) == xb.XCONV_EINVAL
    assert L.xconv_layernorm_fwd(p, odd, None, None, ONE, None, None, None) == xb.XCONV_EINVAL
    assert L.xconv_layernorm_fwd(p, ONE, ctypes.c_void_p(4098), None, ONE, None, None, None) == xb.XCONV_EINVAL
    assert L.xconv_layernorm_fwd(p, ONE, None, None, ONE, ctypes.c_void_p(4098), None, None) == xb.XCONV_EINVAL
    bwd = lambda *a: L.xconv_layernorm_bwd(p, *a, None)
    assert bwd(None, ONE, ONE, ONE, None, ONE, None, None, None, 0) == xb.XCONV_EINVAL
    assert bwd(ONE, ONE, None, ONE, None, ONE, None, None, None, 0) == xb.XCONV_EINVAL
    assert bwd(ONE, ONE, ONE, ONE, None, ONE, ONE, None, None, 1 << 30) == xb.XCONV_EINVAL
    assert bwd(ONE, ONE, ONE, ONE, None, None, None, ONE, ONE, 16) == xb.XCONV_EWORKSPACE
    assert bwd(ONE, ONE, ONE, ONE, None, None, None, None, None, 0) == xb.XCONV_OK          # nothing is wanted
    empty = xb.make_norm_desc(0, 24)
    assert L.xconv_layernorm_fwd(ctypes.byref(empty), None, None, None, None, None, None, None) == xb.XCONV_OK


def test_orth_statuses():
    L = xb.lib()
    items = lambda *m: xb.make_orth_items([(r, c, 4096, 4096, 4096) for r, c in m])
    args = xb.make_orth_args()
    mu = ctypes.byref(xb.xconv_muon_args(0.1, 0.9, 0.0, 1))
    size = xb.xconv_orth_workspace_bytes(items((128, 1152), (10, 3)), 2, args)
    assert size >= 128 * 1152 * 4 and size % 256 == 0
    # the scratch of a long list is that of a launch, not of the list
    many = xb.xconv_orth_workspace_bytes(items(*[(128, 1152)] * 100), 100, args)
    assert size < many < 100 * size

    def both(it, n, a, status, ws=ONE, nbytes=1 << 40):
        pa = ctypes.byref(a) if a is not None else None
        assert L.xconv_orth(it, n, pa, ws, nbytes, None) == status
        assert L.xconv_muon_step(it, n, pa, mu, ws, nbytes, None) == status

    both(items((4, 4)), 0, args, xb.XCONV_OK)
    both(items((4, 4)), -1, args, xb.XCONV_EINVAL)
    both(None, 1, args, xb.XCONV_EINVAL)
    both(items((4, 4)), 1, None, xb.XCONV_EINVAL)
    both(items((4, 4)), 1, args, xb.XCONV_EINVAL, ws=None)
    both(items((4, 4)), 1, args, xb.XCONV_EINVAL, ws=ctypes.c_void_p(4096 + 16))
    both(items((4, 4)), 1, args, xb.XCONV_EWORKSPACE, nbytes=64)
    for bad in ((0, 4), (4, 0), (-1, 4)):
        both(items((4, 4), bad), 2, args, xb.XCONV_EINVAL)
        assert xb.xconv_orth_workspace_bytes(items(bad), 1, args) == 0
    for bad in ((40000, 40000), ((1 << 24) + 1, 2), (1 << 17, 1 << 15)):
        both(items(bad), 1, args, xb.XCONV_EUNSUPPORTED)
    for kw, status in (({"g_dtype": 3}, 1), ({"out_dtype": -1}, 1), ({"steps": -1}, 1), ({"steps": 65}, 2), ({"eps": -1.0}, 1), ({"eps": float("nan")}, 1),
                       ({"coefficients": (float("inf"), 0, 0)}, 1), ({"coefficients": (13.0, 0, 0)}, 2), ({"coefficients": (4.0, 0, 0)}, 2),
                       ({"coefficients": (1.5, 0.5, 0.0), "steps": 20}, 2), ({"coefficients": (1.0, 40.0, -40.0)}, 2)):
        both(items((4, 4)), 1, xb.make_orth_args(**kw), status)
    # a last step may end anywhere: only what is split into fp16 numbers is bounded
    assert xb.xconv_orth_workspace_bytes(items((4, 4)), 1, xb.make_orth_args(coefficients=(4.0, 0, 0), steps=1)) > 0
    assert L.xconv_muon_step(items((4, 4)), 1, ctypes.byref(args), None, ONE, 1 << 30, None) == xb.XCONV_EINVAL
    assert L.xconv_muon_step(items((4, 4)), 1, ctypes.byref(args), ctypes.byref(xb.xconv_muon_args(float("nan"), 0.9, 0, 1)), ONE, 1 << 30, None) == xb.XCONV_EINVAL
    no_m = xb.make_orth_items([(4, 4, 4096, 4096, None)])
    assert L.xconv_muon_step(no_m, 1, ctypes.byref(args), mu, ONE, 1 << 30, None) == xb.XCONV_EINVAL
    odd = xb.make_orth_items([(4, 4, 4098, 4096, None)])
    assert L.xconv_orth(odd, 1, ctypes.byref(args), ONE, 1 << 30, None) == xb.XCONV_EINVAL


def test_python_refusals_without_a_gpu():
    x = torch.zeros(3, 4)
    for call in (lambda: norm.layer_norm(x), lambda: norm.layer_norm_forward(x), lambda: norm.layer_norm_backward(x, x, x, x), lambda: optim.orthogonalize(x),
                 lambda: optim.muon_step([x], [x], [x], 0.1)):
        with pytest.raises(RuntimeError, match="GPU only"):
            call()
    assert optim.orthogonalize([]) == [] and optim.muon_step([], [], [], 0.1) is None
    with pytest.raises(ValueError):
        optim.muon_step([], [x], [], 0.1)
    with pytest.raises(TypeError):
        optim.orthogonalize([3])
    for kw in ({"channels": 0}, {"channels": 4, "axis": 2}, {"channels": 4, "eps": -1.0}, {"channels": 4, "eps": float("nan")}):
        with pytest.raises(ValueError):
            norm.XLayerNorm(**kw)
    w = torch.nn.Parameter(torch.zeros(3, 4))
    for kw in ({"lr": -1}, {"momentum": 1.5}, {"weight_decay": -1}, {"steps": 1.5}, {"coefficients": (1, 2)}, {"eps": -1.0}):
        with pytest.raises(ValueError):
            optim.Muon([w], **kw)
    with pytest.raises(ValueError, match="two and more axes"):
        optim.Muon([torch.nn.Parameter(torch.zeros(3))])
    optim.Muon([w]).step()                # no gradient: nothing to do
