"""Sizes of 4-bit weights that are refused before any device work."""
import ctypes

from test_host_q4 import L, UNSUPPORTED, fake, ll  # noqa: F401


def test_weight_rows(L):  # noqa: F811
    h = ctypes.c_void_p()
    for k in (2 ** 27 - 15, 2 ** 31 - 1):
        assert L.fscnn_q4_compress(fake, 1, k, 8, ll(8), 128, 0, None, ctypes.byref(h)) == UNSUPPORTED
        assert L.fscnn_q4_import(fake, fake, 1, None, k, 8, 128, None, ctypes.byref(h)) == UNSUPPORTED
    assert not h.value
