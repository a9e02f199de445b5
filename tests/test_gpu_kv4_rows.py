"""GPU tests of the 4-bit cache's rows: what hdf_kv4_write_rows stores and hdf_kv4_read_rows returns,
against the oracle.  Codes and scales are decided without error, so what is read is compared for
equality: keys are exact in both types, a value is code * scale rounded once to the type."""
import numpy as np
import pytest
import torch

from oracle import kv4 as ref
from paper_2606_26744_amd import hdf

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


def _expect(k, v, nh, hd, dtype):
    n = k.shape[0]
    kd = ref.quantise_keys(_np(k).reshape(n, nh, hd)).reshape(n, -1)
    vd = ref.quantise_values(_np(v).reshape(n, nh, hd)).reshape(n, -1)
    cast = lambda x: torch.from_numpy(x).to(dtype).float().numpy().astype(np.float64)
    return cast(kd), cast(vd)


def _same(got, want):
    got = _np(got)
    assert np.array_equal(got, want, equal_nan=True), \
        (np.argwhere(~((got == want) | (np.isnan(got) & np.isnan(want))))[:5],)


def _rows(n, width, dtype, seed, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    size = torch.exp(2 * torch.randn(n, 1, generator=g, device="cuda"))
    wide = torch.zeros(n, width + pad, dtype=dtype, device="cuda")
    wide[:, :width] = (torch.randn(n, width, generator=g, device="cuda") * size).to(dtype)
    return wide[:, :width]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,row0", [(1, 0), (1, 77), (7, 3), (8, 8), (150, 61), (64, 64)])
def test_runs(hd, dtype, n, row0):
    nh, cap = 3, 256
    kv4 = hdf.kv4_alloc(2, nh, hd, cap)
    k, v = _rows(n, nh * hd, dtype, 1), _rows(n, nh * hd, dtype, 2, pad=16)
    hdf.kv4_write_rows(kv4, 1, k, v, row0=row0)
    want = _expect(k, v, nh, hd, dtype)
    for got, w in zip(hdf.kv4_read_rows(kv4, 1, n, row0=row0, dtype=dtype), want):
        _same(got, w)
    # Everything else is still zero: rows around, and the other layer.
    for layer, rows in ((1, [r for r in range(cap) if not row0 <= r < row0 + n]), (0, range(cap))):
        at = torch.tensor(list(rows), dtype=torch.int32, device="cuda")
        for got in hdf.kv4_read_rows(kv4, layer, len(at), rows=at, dtype=F32):
            assert not got.any()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_lists(hd, dtype):
    """Scattered rows, runs across words, whole words, rows outside the cache."""
    nh, cap = 2, 192
    kv4 = hdf.kv4_alloc(1, nh, hd, cap)
    k0, v0 = _rows(cap, nh * hd, dtype, 3), _rows(cap, nh * hd, dtype, 4)
    hdf.kv4_write_rows(kv4, 0, k0, v0)
    rows = ([5, 6, 7, 8, 9, 10] + list(range(64, 72)) + [191, -1, 100, 192, 98, 101, 103]
            + list(range(16, 24)) + [150, 0, 151, 2**31 - 1, 1])
    n = len(rows)
    at = torch.tensor(rows, dtype=torch.int32, device="cuda")
    k, v = _rows(n, nh * hd, dtype, 5, pad=8), _rows(n, nh * hd, dtype, 6)
    hdf.kv4_write_rows(kv4, 0, k, v, rows=at)
    full = [x.copy() for x in _expect(k0, v0, nh, hd, dtype)]
    part = _expect(k, v, nh, hd, dtype)
    for i, r in enumerate(rows):
        for f, p in zip(full, part):
            if 0 <= r < cap:
                f[r] = p[i]
            else:
                p[i] = 0
    for got, w in zip(hdf.kv4_read_rows(kv4, 0, cap, dtype=dtype), full):
        _same(got, w)
    for got, w in zip(hdf.kv4_read_rows(kv4, 0, n, rows=at, dtype=dtype), part):
        _same(got, w)


def test_keys_or_values_alone():
    nh, hd = 2, 128
    kv4 = hdf.kv4_alloc(1, nh, hd, 64)
    k, v = _rows(30, nh * hd, BF, 7), _rows(30, nh * hd, BF, 8)
    hdf.kv4_write_rows(kv4, 0, k, None, row0=9)
    want = _expect(k, v, nh, hd, BF)
    got = hdf.kv4_read_rows(kv4, 0, 30, row0=9)
    _same(got[0], want[0])
    assert not got[1].any()
    hdf.kv4_write_rows(kv4, 0, None, v, row0=9)
    only = torch.zeros(30, 2 * nh * hd, dtype=BF, device="cuda")
    hdf.kv4_read_rows(kv4, 0, 30, row0=9, out=(None, only[:, nh * hd:]))
    _same(only[:, nh * hd:], want[1])
    assert not only[:, :nh * hd].any()


def _borders(dtype):
    """Elements on and next to every border between codes, at scales of every size."""
    out = []
    for e in (-126, -110, -3, 0, 5, 100, 124):
        for m in (1.0, 1.2890625, 1.9921875):
            s = m * 2.0 ** e
            row = [6 * s]
            for t in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0):
                x = torch.tensor(t * s, dtype=torch.float64).to(dtype)
                near = [x, torch.nextafter(x, x * 2), torch.nextafter(x, x / 2)]
                row += [float(a) * sgn for a in near for sgn in (1, -1)]
            row = [min(max(a, -6 * s), 6 * s) for a in row][:64]
            out.append(row + [0.0] * (64 - len(row)))
    return torch.tensor(out, dtype=torch.float64).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_borders_between_codes(dtype):
    x = _borders(dtype)
    n = x.shape[0]
    x = torch.cat([x, x.flip(1) * 0.5], 1)
    for hd in (64, 128):
        nh = 128 // hd
        kv4 = hdf.kv4_alloc(1, nh, hd, 64)
        hdf.kv4_write_rows(kv4, 0, x, x, row0=2)
        # In 32 bits what the cache stands for is exact.
        for got, w in zip(hdf.kv4_read_rows(kv4, 0, n, row0=2, dtype=F32), _expect(x, x, nh, hd, F32)):
            _same(got, w)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_extremes_and_what_is_no_number(dtype):
    hd, nh = 128, 1
    big = torch.finfo(dtype).max
    x = torch.randn(10, hd, generator=torch.Generator().manual_seed(0)).to(dtype).cuda()
    x[0] = 0
    x[1] = big
    x[2, 3] = -big
    x[3] *= 2.0 ** -126
    x[4] = 2.0 ** -133
    x[5, 70] = float("nan")
    x[6, 5] = float("inf")
    x[7, 127] = -float("inf")
    x[8] = -0.0
    kv4 = hdf.kv4_alloc(1, nh, hd, 64)
    hdf.kv4_write_rows(kv4, 0, x, x, row0=1)
    for got, w in zip(hdf.kv4_read_rows(kv4, 0, 10, row0=1, dtype=F32), _expect(x, x, nh, hd, F32)):
        _same(got, w)


def test_no_rows_and_another_stream():
    kv4 = hdf.kv4_alloc(1, 1, 64, 64)
    none = torch.empty(0, 64, dtype=BF, device="cuda")
    hdf.kv4_write_rows(kv4, 0, none, none)
    assert hdf.kv4_read_rows(kv4, 0, 0)[0].shape == (0, 64)
    k, v = _rows(40, 64, BF, 9), _rows(40, 64, BF, 10)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    hdf.kv4_write_rows(kv4, 0, k, v, stream=side)
    got = hdf.kv4_read_rows(kv4, 0, 40, stream=side)
    side.synchronize()
    for x, w in zip(got, _expect(k, v, 1, 64, BF)):
        _same(x, w)


def test_tiles_beyond_32_bits():
    """A cache of more than 4 GiB: rows of its last tiles, of the last head."""
    nh, hd = 8, 128
    cap = 64 * 66000                    # 8 * 66000 * 8576 bytes
    kv4 = torch.zeros((1, nh, cap // 64, 8576), dtype=torch.uint8, device="cuda")
    assert kv4.numel() > 1 << 32
    k, v = _rows(70, nh * hd, BF, 11), _rows(70, nh * hd, BF, 12)
    hdf.kv4_write_rows(kv4, 0, k, v, row0=cap - 70)
    for x, w in zip(hdf.kv4_read_rows(kv4, 0, 70, row0=cap - 70), _expect(k, v, nh, hd, BF)):
        _same(x, w)
    assert not kv4[:, :, :cap // 64 - 2].any()


def test_a_row_named_twice_disturbs_no_other():
    """What that row then holds is open; its neighbours, whose values share its words, keep theirs."""
    nh, hd, cap = 2, 128, 64
    kv4 = hdf.kv4_alloc(1, nh, hd, cap)
    k0, v0 = _rows(cap, nh * hd, BF, 13), _rows(cap, nh * hd, BF, 14)
    hdf.kv4_write_rows(kv4, 0, k0, v0)
    before = hdf.kv4_read_rows(kv4, 0, cap)
    rows = [3, 3] + list(range(20, 28)) + [3, 40, 3]       # in one wave's eight rows, and in another's
    k, v = _rows(len(rows), nh * hd, BF, 15), _rows(len(rows), nh * hd, BF, 16)
    hdf.kv4_write_rows(kv4, 0, k, v, rows=torch.tensor(rows, dtype=torch.int32, device="cuda"))
    once = [i for i, r in enumerate(rows) if r != 3]
    want = _expect(k[once], v[once], nh, hd, BF)
    for got, old, w in zip(hdf.kv4_read_rows(kv4, 0, cap), before, want):
        _same(got[[rows[i] for i in once]], w)
        rest = [r for r in range(cap) if r not in rows]
        assert torch.equal(got[rest], old[rest])


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_long_reads_are_those_of_their_pieces(hd, dtype):
    """Long reads go by larger workgroups: runs and lists of rows, odd heads, rows outside the cache."""
    nh, n = 33, 8209
    cap = 64 * 130
    kv4 = hdf.kv4_alloc(1, nh, hd, cap)
    hdf.kv4_write_rows(kv4, 0, _rows(cap, nh * hd, dtype, 17), _rows(cap, nh * hd, dtype, 18))
    order = torch.randperm(cap, generator=torch.Generator().manual_seed(3))[:n].int()
    order[::1000] = -1
    order[5::1000] = cap
    order[80:96] = torch.arange(80, 96, dtype=torch.int32)
    order = order.cuda()
    for kw in (dict(row0=13), dict(rows=order)):
        got = hdf.kv4_read_rows(kv4, 0, n, dtype=dtype, **kw)
        for lo in range(0, n, 1000):
            m = min(1000, n - lo)
            part = dict(row0=13 + lo) if "row0" in kw else dict(rows=order[lo:lo + m].contiguous())
            for x, y in zip(got, hdf.kv4_read_rows(kv4, 0, m, dtype=dtype, **part)):
                assert torch.equal(x[lo:lo + m], y), lo
