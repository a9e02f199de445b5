"""Refusals of the truncated-distribution calls, before any device is touched."""
import ctypes

import pytest
import torch

from paper_2606_26744_amd import hdf

FAKE = ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4098)


def _params(**kw):
    p = hdf.TruncationParams(1.0, 0, 1.0, 0.0, None, None, None, None, 1)
    for k, v in kw.items():
        setattr(p, k, v)
    return ctypes.byref(p)


def _status(st):
    return hdf.STATUS[st]


def _sample(rows=4, V=100, ld=100, dtype=0, params=None, logits=FAKE, u=FAKE, tok=FAKE, kept=FAKE,
            ws=FAKE, ws_bytes=1 << 30):
    return _status(hdf.lib().hdf_sample_truncated(
        logits, rows, V, ld, dtype, params if params is not None else _params(), u, tok, kept, FAKE,
        FAKE, FAKE, ws, ws_bytes, None))


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(V=0), dict(ld=99), dict(dtype=3), dict(logits=None), dict(kept=None),
    dict(u=None), dict(tok=None), dict(logits=ODD),
    dict(params=_params(temperature=-0.1)), dict(params=_params(temperature=float("inf"))),
    dict(params=_params(temperature=float("nan"))), dict(params=_params(top_k=-1)),
    dict(params=_params(top_p=-0.5)), dict(params=_params(top_p=float("nan"))),
    dict(params=_params(min_p=1.5)), dict(params=_params(min_p=-0.1)),
    dict(params=_params(rows_per_seq=0))])
def test_sample_invalid(kw):
    assert _sample(**kw) == "HDF_E_INVALID"


def test_sample_limits():
    assert _sample(rows=65536) == "HDF_E_UNSUPPORTED"
    assert _sample(V=(1 << 20) + 1, ld=1 << 21) == "HDF_E_UNSUPPORTED"
    assert _sample(rows=0, logits=None, kept=None, u=None, tok=None, ws=None, ws_bytes=0) == "HDF_OK"
    L = hdf.lib()
    assert _status(L.hdf_sample_truncated(FAKE, 4, 100, 100, 0, None, FAKE, FAKE, FAKE, FAKE, FAKE,
                                          FAKE, FAKE, 1 << 30, None)) == "HDF_E_INVALID"


def _accept(stride=15, draft_dtype=0, ld=100, target_dtype=0, n_seq=2, K=15, V=100, params=None,
            draft=FAKE, dcl=FAKE, target=FAKE, u=FAKE, acc=FAKE, ws=FAKE, ws_bytes=1 << 30):
    return _status(hdf.lib().hdf_accept_truncated(
        draft, stride, FAKE, draft_dtype, ld, dcl, FAKE, FAKE, target, target_dtype, n_seq, K, V,
        params if params is not None else _params(), u, acc, FAKE, None, None, ws, ws_bytes, None))


@pytest.mark.parametrize("kw", [
    dict(n_seq=-1), dict(K=-1), dict(K=1025, stride=1025), dict(stride=14), dict(ld=99), dict(V=0),
    dict(draft_dtype=2), dict(target_dtype=2), dict(draft=None), dict(dcl=None), dict(target=None),
    dict(u=None), dict(acc=None), dict(params=_params(top_k=-1)), dict(ws=ctypes.c_void_p(4100))])
def test_accept_invalid(kw):
    assert _accept(**kw) == "HDF_E_INVALID"


def test_accept_limits_and_workspace():
    assert _accept(n_seq=4096) == "HDF_E_UNSUPPORTED"            # 65536 target rows
    assert _accept(V=(1 << 20) + 1, ld=1 << 21) == "HDF_E_UNSUPPORTED"
    assert _accept(n_seq=0, draft=None, target=None, u=None, acc=None, ws=None) == "HDF_OK"
    L = hdf.lib()
    need = L.hdf_accept_truncated_workspace(2, 15, 100, 0)
    assert need > 0
    assert _accept(ws_bytes=need - 1) == "HDF_E_WORKSPACE"
    assert _accept(ws=None) == "HDF_E_WORKSPACE"
    for bad in ((-1, 15, 100, 0), (2, 1025, 100, 0), (2, 15, 0, 0), (2, 15, 100, 7),
                (4096, 15, 100, 0)):
        assert L.hdf_accept_truncated_workspace(*bad) == 0
    # a workspace for more sequences serves fewer
    sizes = [L.hdf_accept_truncated_workspace(n, 15, 4097, 1) for n in range(1, 70)]
    assert sizes == sorted(sizes)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("V", [1, 100, 4097, 32003, 129280, 262145, 1 << 20])
def test_workspaces_serve_fewer_rows(V, dtype):
    """The need of every smaller call lies within the size that is reported for a larger one."""
    L = hdf.lib()
    rows = list(range(1, 300)) + list(range(300, 9000, 131)) + [65535]
    for size in (lambda n: L.hdf_sample_truncated_workspace(n, V, dtype),
                 lambda n: L.hdf_top_logits_workspace(n, V, 5, dtype)):
        sizes = [size(n) for n in rows]
        assert sizes[0] > 0 and sizes == sorted(sizes)


def _top(rows=4, V=100, ld=100, dtype=0, K=5, T=1.0, logits=FAKE, ids=FAKE, values=FAKE):
    return _status(hdf.lib().hdf_top_logits(logits, rows, V, ld, dtype, K, T, ids, values, None,
                                            FAKE, 1 << 30, None))


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(V=0), dict(ld=99), dict(dtype=3), dict(K=0), dict(K=1025), dict(T=0.0),
    dict(T=float("inf")), dict(T=float("nan")), dict(logits=None), dict(ids=None),
    dict(values=None)])
def test_top_invalid(kw):
    assert _top(**kw) == "HDF_E_INVALID"


def test_top_limits():
    assert _top(rows=65536) == "HDF_E_UNSUPPORTED"
    assert _top(V=(1 << 20) + 1, ld=1 << 21) == "HDF_E_UNSUPPORTED"
    assert _top(rows=0, logits=None, ids=None, values=None) == "HDF_OK"


def test_binding_refuses_host_tensors_and_bad_shapes():
    z = torch.zeros(4, 10)
    for call in (lambda: hdf.sample_truncated(z), lambda: hdf.top_logits(z, 3),
                 lambda: hdf.sample_truncated(torch.zeros(10)),
                 lambda: hdf.sample_truncated(torch.zeros(10, 4).t()),
                 lambda: hdf.top_logits(torch.zeros(1, 10).expand(4, 10), 3),
                 lambda: hdf.sample_truncated(z, rows_per_seq=0),
                 lambda: hdf.sample_truncated(z, top_p=torch.ones(3)),
                 lambda: hdf.sample_truncated(z, top_k=torch.ones(4)),
                 lambda: hdf.accept_truncated(z, z, (z, z, z, z), z, z, K=3, draft_stride=4)):
        with pytest.raises(ValueError):
            call()
