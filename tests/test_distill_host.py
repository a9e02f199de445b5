"""Refusals of the distillation calls, before any device is touched."""
import ctypes

import pytest
import torch

from paper_2606_26744_amd import hdf
from paper_2606_26744_amd.distill import distill_loss

FAKE = ctypes.c_void_p(4096)
OTHER = ctypes.c_void_p(8192)
ODD = ctypes.c_void_p(4098)


def _status(st):
    return hdf.STATUS[st]


def _fwd(z=FAKE, ld=100, dtype=0, V=100, n=2, B=8, P=3, ids=FAKE, tl=FAKE, K=5, labels=FAKE, T=1.0,
         alpha=0.5, kl=FAKE, ce=FAKE, loss=FAKE, saved=FAKE, ws=FAKE, ws_bytes=1 << 30):
    return _status(hdf.lib().hdf_distill_forward(z, ld, dtype, V, n, B, P, ids, tl, None, K, labels,
                                                 T, alpha, kl, ce, loss, saved, ws, ws_bytes, None))


def _bwd(z=FAKE, ld=100, dtype=0, V=100, n=2, B=8, P=3, ids=FAKE, K=5, labels=FAKE, T=1.0, alpha=0.5,
         saved=FAKE, d=OTHER, ldd=100):
    return _status(hdf.lib().hdf_distill_backward(z, ld, dtype, V, n, B, P, ids, K, labels, T, alpha,
                                                  saved, None, None, None, d, ldd, None))


SHARED = [dict(z=None), dict(ld=99), dict(dtype=5), dict(V=0), dict(n=-1), dict(B=1), dict(B=1026),
          dict(P=0), dict(P=8), dict(ids=None), dict(K=0), dict(K=1025), dict(T=0.0), dict(T=-1.0),
          dict(T=float("nan")), dict(T=1e31), dict(T=1e-31), dict(alpha=float("inf")), dict(z=ODD),
          dict(saved=None), dict(saved=ctypes.c_void_p(4100))]


@pytest.mark.parametrize("kw", SHARED + [dict(tl=None), dict(kl=None), dict(ce=None),
                                         dict(labels=None), dict(loss=None),
                                         dict(ws=ctypes.c_void_p(4100))])
def test_forward_invalid(kw):
    assert _fwd(**kw) == "HDF_E_INVALID"


@pytest.mark.parametrize("kw", SHARED + [dict(d=None), dict(d=FAKE), dict(ldd=99), dict(d=ODD)])
def test_backward_invalid(kw):
    assert _bwd(**kw) == "HDF_E_INVALID"


def test_limits_workspaces_and_empty_batches():
    assert _fwd(n=8192) == "HDF_E_UNSUPPORTED"
    assert _bwd(n=8192) == "HDF_E_UNSUPPORTED"
    assert _fwd(V=(1 << 20) + 1, ld=1 << 21) == "HDF_E_UNSUPPORTED"
    L = hdf.lib()
    need = L.hdf_distill_workspace(2, 8, 100, 0)
    assert need > 0 and _fwd(ws_bytes=need - 1) == "HDF_E_WORKSPACE"
    assert _fwd(ws=None) == "HDF_E_WORKSPACE"
    assert _fwd(n=0, z=None, ids=None, saved=None, ws=None) == "HDF_OK"
    assert _bwd(n=0, z=None, ids=None, saved=None, d=None) == "HDF_OK"
    assert L.hdf_distill_saved_bytes(2, 8, 3, 5) > 0
    for bad in ((-1, 8, 3, 5), (2, 1, 1, 5), (2, 8, 8, 5), (2, 8, 3, 0), (2, 8, 3, 1025)):
        assert L.hdf_distill_saved_bytes(*bad) == 0
    for bad in ((-1, 8, 100, 0), (2, 8, 0, 0), (2, 8, 100, 4)):
        assert L.hdf_distill_workspace(*bad) == 0


def test_binding_refuses_host_tensors_and_bad_shapes():
    z = torch.zeros(8, 10)
    ids, val = torch.zeros(2, 3, 5, dtype=torch.int32), torch.zeros(2, 3, 5)
    for call in (lambda: hdf.distill_forward(z, ids, val, B=4),
                 lambda: hdf.distill_forward(z, ids, val, B=5),
                 lambda: hdf.distill_forward(z, ids.long(), val, B=4),
                 lambda: hdf.distill_forward(z, ids[0], val, B=4),
                 lambda: hdf.distill_forward(z, ids, val[:1], B=4),
                 lambda: hdf.distill_forward(z.t(), ids, val, B=4),
                 lambda: distill_loss(z, ids, val, B=4)):
        with pytest.raises(ValueError):
            call()
