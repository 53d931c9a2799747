"""Host side of the Muon step of 64-bit parameters and of the optimiser, without a GPU."""
import ctypes

from paper_2106_06998_amd import binding as xb

ONE = ctypes.c_void_p(4096)          # never dereferenced: validation fails first


def test_parameters_of_64_bits():
    assert ctypes.sizeof(xb.xconv_muon_args64) == 32 and xb.xconv_muon_args64.nesterov.offset == 24
    L, args = xb.lib(), xb.make_orth_args()
    items = xb.make_orth_items([(4, 4, 4096, 4096, 4096)])
    step = lambda mu, ws=ONE, n=1: L.xconv_muon_step64(items, n, ctypes.byref(args), mu, ws, 1 << 30, None)
    assert step(None) == xb.XCONV_EINVAL
    good = ctypes.byref(xb.xconv_muon_args64(0.1, 0.9, 0.0, 1))
    assert step(good, ws=None) == xb.XCONV_EINVAL and step(good, n=0) == xb.XCONV_OK
    for bad in (float("nan"), float("inf"), 1e300):          # (1e300 is no float)
        for k in range(3):
            v = [0.1, 0.9, 0.0]
            v[k] = bad
            assert step(ctypes.byref(xb.xconv_muon_args64(*v, 1))) == xb.XCONV_EINVAL, (bad, k)
