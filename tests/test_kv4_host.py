"""Host-side checks of the 4-bit cache's calls (no GPU): sizes, refusals before any launch, no-ops."""
import ctypes

import pytest
import torch

from paper_2606_26744_amd import hdf

F = ctypes.c_void_p(4096)      # never dereferenced
BAD = ctypes.c_void_p(4104)    # not 16-byte aligned


def _st(st):
    return hdf.STATUS[st]


def test_sizes():
    L = hdf.lib()
    assert L.hdf_kv4_tile_bytes(128) == 8576 and L.hdf_kv4_tile_bytes(64) == 4352
    assert L.hdf_kv4_tile_bytes(96) == 0
    assert L.hdf_kv4_cache_bytes(2, 8, 128, 640) == 2 * 8 * 10 * 8576
    for bad in ((0, 8, 128, 64), (1, 0, 128, 64), (1, 1, 80, 64), (1, 1, 64, 100), (1, 1, 64, -64),
                (1, 1, 64, 1 << 31), (1 << 30, 1 << 30, 64, 1 << 20)):
        assert L.hdf_kv4_cache_bytes(*bad) == 0, bad
    assert hdf.kv4_alloc(2, 3, 64, 128, device="cpu").shape == (2, 3, 2, 4352)
    for bad in ((1, 1, 96, 64), (1, 1, 64, 65)):
        with pytest.raises(ValueError):
            hdf.kv4_alloc(*bad, device="cpu")


def test_rows_validation():
    L = hdf.lib()

    def w(n=10, rows=None, row0=0, layer=0, nh=2, hd=64, dt=1, kv4=F, cap=128, k=F, v=F, ldk=128, ldv=128):
        return _st(L.hdf_kv4_write_rows(k, ldk, v, ldv, n, rows, row0, layer, nh, hd, dt, kv4, cap, None))

    def r(n=10, rows=None, row0=0, layer=0, nh=2, hd=64, dt=1, kv4=F, cap=128, k=F, v=F, ldk=128, ldv=128):
        return _st(L.hdf_kv4_read_rows(kv4, cap, layer, nh, hd, dt, rows, row0, n, k, ldk, v, ldv, None))
    for call in (w, r):
        for bad in (dict(n=-1), dict(row0=-1), dict(layer=-1), dict(nh=0), dict(dt=3), dict(cap=100),
                    dict(cap=0), dict(row0=120), dict(row0=1 << 40), dict(row0=(1 << 63) - 4), dict(kv4=None),
                    dict(k=None, v=None), dict(k=BAD), dict(v=BAD), dict(kv4=BAD), dict(ldk=127),
                    dict(ldv=64), dict(ldk=132), dict(ldv=1 << 62), dict(ldk=-128), dict(dt=0, ldk=130)):
            assert call(**bad) == "HDF_E_INVALID", bad
        assert call(hd=96) == "HDF_E_UNSUPPORTED"
        assert call(n=1 << 31, rows=F) == "HDF_E_UNSUPPORTED"
        assert call(cap=1 << 31) == "HDF_E_UNSUPPORTED"
        assert call(n=0, k=None, v=None, kv4=None) == "HDF_OK"


def _attend(n_seq=2, B=4, H=8, nkv=2, hd=64, dt=1, cache="paged", max_ctx=100, scale=0.125, q=F, k=F,
            v=F, out=F, ctx=F, blen=None, ldq=512, ldk=128, ldv=128, ldo=512, ws=F, ws_bytes=1 << 40,
            cap=640, layer=0, max_pages=2, kv4=4096):
    c = {"paged": hdf.Kv4Cache(kv4, cap, layer, None, 4096, max_pages),
         "slots": hdf.Kv4Cache(kv4, cap, layer, 4096, None, 0),
         "both": hdf.Kv4Cache(kv4, cap, layer, 4096, 4096, max_pages),
         "neither": hdf.Kv4Cache(kv4, cap, layer, None, None, 0), "none": None}[cache]
    return _st(hdf.lib().hdf_block_attention_kv4(
        q, ldq, k, ldk, v, ldv, n_seq, B, H, nkv, hd, dt, ctypes.byref(c) if c else None, ctx, max_ctx,
        blen, 0, scale, out, ldo, None, ws, ws_bytes, None))


@pytest.mark.parametrize("bad", [
    dict(dt=2), dict(n_seq=-1), dict(max_ctx=-1), dict(B=0), dict(B=65), dict(H=0), dict(nkv=0),
    dict(nkv=3), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38),
    dict(q=None), dict(out=None), dict(ctx=None), dict(k=None), dict(v=None), dict(q=BAD), dict(k=BAD),
    dict(out=BAD), dict(ldq=511), dict(ldq=516), dict(ldo=504), dict(ldk=64), dict(ldv=132),
    dict(ldq=1 << 62), dict(cache="none"), dict(cache="both"), dict(cache="neither"), dict(kv4=None),
    dict(kv4=4104), dict(cap=0), dict(cap=100), dict(cap=-64), dict(cap=1 << 31), dict(layer=-1),
    dict(max_pages=1), dict(max_pages=-1), dict(ws=ctypes.c_void_p(4096 + 16))])
def test_attention_refuses(bad):
    assert _attend(**bad) == "HDF_E_INVALID"


def test_attention_limits_and_no_ops():
    for bad in (dict(hd=96), dict(n_seq=65536), dict(n_seq=40000, B=16), dict(nkv=65536, H=65536),
                dict(max_ctx=(1 << 30) + 1, max_pages=1 << 25)):
        assert _attend(**bad) == "HDF_E_UNSUPPORTED", bad
    assert _attend(max_ctx=100000, max_pages=2000, ws=None, ws_bytes=0) == "HDF_E_WORKSPACE"
    assert _attend(max_ctx=100000, max_pages=2000, ws_bytes=64) == "HDF_E_WORKSPACE"
    assert _attend(n_seq=0, q=None, out=None, ctx=None, k=None, v=None, cache="none") == "HDF_OK"


def test_a_workspace_serves_every_shorter_context():
    size = hdf.lib().hdf_block_attention_kv4_workspace
    for n_seq, B, H, nkv in ((1, 1, 32, 8), (1, 64, 64, 1), (3, 5, 6, 6), (64, 16, 32, 32), (1, 1, 1, 1)):
        for hd in (64, 128):
            last = 0
            for ctx in list(range(0, 9000, 37)) + [1 << k for k in range(14, 31)]:
                need = size(n_seq, B, H, nkv, hd, ctx)
                assert need >= last, (n_seq, B, H, nkv, hd, ctx)
                last = need
    assert size(1, 0, 1, 1, 64, 10) == 0 and size(1, 1, 3, 2, 64, 10) == 0


def test_binding_refuses_tensors_of_other_shapes_and_types():
    kv4 = hdf.kv4_alloc(1, 2, 64, 128, device="cpu")
    rows = torch.zeros(3, 128)
    for bad in (rows[:, ::2], rows[:, :64], rows[0], torch.zeros(3, 129)[:, :127]):
        with pytest.raises(ValueError):
            hdf.kv4_write_rows(kv4, 0, bad, None)
    for kw in (dict(layer=1), dict(layer=-1), dict(rows=torch.zeros(2, dtype=torch.int32)),
               dict(rows=torch.zeros(3, dtype=torch.int64)), dict(row0=-1), dict(row0=1 << 40)):
        layer = kw.pop("layer", 0)
        with pytest.raises(ValueError):
            hdf.kv4_write_rows(kv4, layer, rows, None, **kw)
    with pytest.raises(ValueError):
        hdf.kv4_write_rows(kv4, 0, None, None)
    with pytest.raises(ValueError):
        hdf.kv4_write_rows(kv4, 0, rows, rows.bfloat16())
    with pytest.raises(ValueError):       # a host tensor
        hdf.kv4_write_rows(kv4, 0, rows, rows)
    with pytest.raises(ValueError):
        hdf.kv4_read_rows(kv4, 0, -1)
    for bad in (kv4[..., :100], kv4[:, :, ::2], kv4.float(), kv4[0]):
        with pytest.raises(ValueError):
            hdf.kv4_read_rows(bad, 0, 1)
    q = torch.zeros(1, 4, 2, 64)
    i32 = torch.zeros(2, dtype=torch.int32)
    ok = dict(ctx_len=i32, max_ctx=64, kv_offsets=i32)
    for kw in (dict(ok, ctx_len=i32.long()), dict(ok, kv_offsets=None), dict(ok, page_table=i32.view(1, 2)),
               dict(ok, k_blk=q), dict(ok, k_blk=q, v_blk=q[:, :, :1]), dict(ok, max_ctx=1 << 33),
               dict(ok, k_blk=q.bfloat16(), v_blk=q.bfloat16()), dict(ok, block_len=i32[:0])):
        with pytest.raises(ValueError):
            hdf.block_attention_kv4(q, kv4, 0, **kw)
    for bad in (q[0], torch.zeros(1, 4, 2, 128)):
        with pytest.raises(ValueError):
            hdf.block_attention_kv4(bad, kv4, 0, **ok)
    with pytest.raises(TypeError):
        hdf.block_attention_kv4(q.half(), kv4, 0, **ok)
    for bad in (torch.zeros(2, 4, 2, 128)[..., :64], torch.zeros(2, 5, 2, 64)[:, :4],
                torch.zeros(2, 4, 2, 128)[..., ::2]):
        with pytest.raises(ValueError):
            hdf._block_stride(bad, (2, 4, 2, 64), "q")
    wide = torch.zeros(2, 4, 512)[..., :128].view(2, 4, 2, 64)
    assert hdf._block_stride(wide, (2, 4, 2, 64), "q") == 512
    assert hdf._block_stride(wide[:1, :1], (1, 1, 2, 64), "q") == 128


def test_draft_block_validation():
    from tests.test_abi import _fake_drafter
    L = hdf.lib()
    w, keep = _fake_drafter()

    def call(n_seq=2, B=16, max_ctx=100, counts=None, n_new=8, offs=None, table=F, max_pages=4, kv4=F,
             cap=640, ws=F, ws_bytes=1 << 40, hidden=F):
        return _st(L.hdf_draft_block_kv4(ctypes.byref(w), n_seq, B, F, max_ctx, F, F, counts, n_new, offs,
                                         table, max_pages, kv4, cap, F, hidden, ws, ws_bytes, None))
    for bad in (dict(offs=F), dict(table=None), dict(table=None, offs=F, counts=F), dict(max_pages=1),
                dict(max_pages=-1), dict(kv4=None), dict(cap=100), dict(cap=-64), dict(B=65), dict(B=0),
                dict(n_seq=-1), dict(max_ctx=-1), dict(n_new=-1), dict(kv4=BAD), dict(hidden=None),
                dict(ws=ctypes.c_void_p(4112))):
        assert call(**bad) == "HDF_E_INVALID", bad
    assert call(n_seq=70000) == "HDF_E_UNSUPPORTED"
    assert call(ws=None, ws_bytes=0) == "HDF_E_WORKSPACE"
    assert call(ws_bytes=1000) == "HDF_E_WORKSPACE"
    assert call(n_seq=0) == "HDF_OK"
    size = L.hdf_draft_block_kv4_workspace
    last = 0
    for n_new in list(range(0, 400, 13)) + [2048, 2049, 16384, 16385, 20000]:
        need = size(ctypes.byref(w), 8, 16, n_new, 5000)
        assert need >= last
        last = need
    assert size(ctypes.byref(w), 70000, 16, 0, 10) == 0 and size(None, 1, 1, 0, 10) == 0
