"""Gradients that share memory with the logits, which are read after other columns' gradients were
written, are refused before any device is touched."""
import ctypes

import pytest

from paper_2606_26744_amd import hdf

Z, WS = 1 << 20, 1 << 32


def _bwd(d, ld=100, ldd=100, dtype=0, V=100, n=2, B=8):
    return hdf.STATUS[hdf.lib().hdf_distill_backward(
        ctypes.c_void_p(Z), ld, dtype, V, n, B, 3, ctypes.c_void_p(WS), 5, ctypes.c_void_p(WS), 1.0, 0.5,
        ctypes.c_void_p(WS), None, None, None, ctypes.c_void_p(d), ldd, None)]


@pytest.mark.parametrize("dtype,size", [(0, 4), (1, 2)])
def test_rows_that_meet(dtype, size):
    for ld, ldd in ((100, 100), (300, 300), (300, 100), (100, 301), (157, 211)):
        # The first, a middle and the last row; whole, and the first and last element alone.
        for r, s in ((0, 0), (15, 0), (0, 15), (7, 7), (3, 8)):
            for off in (0, 1, 99, -1, -99):
                d = Z + (r * ld + off) * size - s * ldd * size
                assert _bwd(d, ld, ldd, dtype) == "HDF_E_INVALID", (ld, ldd, r, s, off)
                assert "share memory" in hdf.lib().hdf_last_error().decode()

