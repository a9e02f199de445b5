"""GPU tests of hdf_block_attention_kv4 against the oracle over what the cache stands for.

Bound of an output element, with A = sum p |v| (at least |out|):
  a score is off by d <= (hd + 4) 2^-24 scale sum |q k| + 2^-22 (fp32 sums; the exponential and
  its argument; bf16: the argument holds a power of two of up to 2^94, half a step 2^-18), its
  probability by a factor 1 + d, the ratio of sums by 2 d; bf16: a probability
  times its value's scale is rounded to fp16, 2^-11 of itself, or 2^-25 in units of 2^-11 of the
  greatest probability (at most 1 of the sum) times twice the greatest scale, so 2^-35 max |v| a key
  (the reference of the probabilities is at most 2^4 below the greatest, and their factor's top 2^15);
  fp32: a probability in three bf16 terms, 2^-24, a query in three, 2^-24 more of its score; sums
  over T keys in fp32, each at most T 2^-24; the result is rounded once, 2^-8 of itself (bf16) or
  2^-24 (fp32).  What lies below fp32's least normal number, 2^-126, may be 0: a key's probability
  relative to the greatest and the lower term it is split into, so 2 * 2^-126 max |v| a key.
"""
import numpy as np
import pytest
import torch

from oracle import kv4 as ref
from paper_2606_26744_amd import hdf

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


class Case:
    def __init__(self, ctx, B, H, nkv, hd, dtype, *, paged=True, block=True, fused=False, seed=0,
                 layers=1, layer=0, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        n = len(ctx)
        self.ctx, self.B, self.H, self.nkv, self.hd, self.dtype, self.layer = ctx, B, H, nkv, hd, dtype, layer
        tiles = [(t + 63) // 64 for t in ctx]
        total = sum(tiles) + 2
        order = torch.randperm(total, generator=g).tolist()
        self.kv4 = hdf.kv4_alloc(layers, nkv, hd, 64 * total)
        self.kv4.fill_(0xFF)            # rows that no sequence holds: NaN scales
        self.max_ctx = max(max(ctx), 1)
        width = max((self.max_ctx + 63) // 64, 1)
        table, offs, at = np.full((n, width), -1, np.int32), [0], 0
        self.k, self.v = [], []
        for s, T in enumerate(ctx):
            pages = order[at:at + tiles[s]] if paged else list(range(at, at + tiles[s]))
            at += tiles[s]
            table[s, :tiles[s]] = pages
            offs.append(64 * at)
            k = torch.randn(T, nkv, hd, generator=g) * spread
            v = torch.randn(T, nkv, hd, generator=g) * torch.exp(torch.randn(T, nkv, 1, generator=g))
            k, v = k.to(dtype), v.to(dtype)
            if T:
                hdf.kv4_write_rows(self.kv4, layer, k.view(T, -1).cuda(), v.view(T, -1).cuda(),
                                   rows=hdf.paged_rows(pages, T, "cuda"))
            self.k.append(ref.quantise_keys(_np(k)))
            self.v.append(ref.quantise_values(_np(v)))
        i32 = dict(dtype=torch.int32, device="cuda")
        self.kw = dict(ctx_len=torch.tensor(ctx, **i32), max_ctx=self.max_ctx)
        if paged:
            self.kw["page_table"] = torch.from_numpy(table).cuda()
        else:
            self.kw["kv_offsets"] = torch.tensor(offs, **i32)
        wide = (torch.randn(n, B, (H + 2 * nkv) * hd, generator=g) * spread).to(dtype).cuda()
        cols = wide[..., :H * hd], wide[..., H * hd:(H + nkv) * hd], wide[..., (H + nkv) * hd:]
        cols = [c if fused else c.contiguous() for c in cols]
        self.q = cols[0].view(n, B, H, hd)
        self.kb, self.vb = (c.view(n, B, nkv, hd) for c in cols[1:])
        if block:
            self.kw.update(k_blk=self.kb, v_blk=self.vb)
        self.block = block

    def check(self, out, lse, *, causal=False, blen=None, scale=None):
        f32 = self.dtype == F32
        for s, T in enumerate(self.ctx):
            b = self.B if blen is None else blen[s]
            kb, vb = (_np(self.kb[s, :b]), _np(self.vb[s, :b])) if self.block else (None, None)
            o, l, mass, reach = ref.attend(_np(self.q[s, :b]), self.k[s], self.v[s], kb, vb,
                                           causal=causal, scale=scale)
            d = (self.hd + 4) * 2.0 ** -24 * reach + 2.0 ** -22 + (2.0 ** -24 * reach if f32 else 2.0 ** -18)
            N = T + self.B
            tol = mass * (2 * d[..., None] + (2.0 ** -24 if f32 else 2.0 ** -11) + 2 * N * 2.0 ** -24)
            tol += np.abs(o) * (2.0 ** -24 if f32 else 2.0 ** -8)
            top = max([np.abs(x).max() for x in (self.v[s], vb) if x is not None and x.size] or [0.0])
            tol += N * (2 * 2.0 ** -126 + (0 if f32 else 2.0 ** -35)) * top
            tol += N * 6 * 2.0 ** -120
            err = np.abs(_np(out[s, :b]) - o)
            assert (err <= tol).all(), (s, T, float((err - tol).max()), np.argwhere(err > tol)[:3])
            if lse is not None:
                got = _np(lse[s, :b])
                fin = np.isfinite(l)
                assert np.array_equal(got[~fin], l[~fin])
                e = np.abs(got[fin] - l[fin])
                bound = (d + N * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(l)))[fin]
                assert (e <= bound).all(), (s, T, float((e - bound).max()))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,nkv", [(1, 4, 4), (16, 2, 2), (5, 6, 3), (16, 8, 2), (33, 2, 1), (1, 14, 2)])
def test_blocks_over_ragged_contexts(hd, dtype, B, H, nkv):
    print(f"[kv4 attention] hd={hd} {dtype} B={B} H={H}/{nkv}", flush=True)
    c = Case([1, 64, 130, 0, 700], B, H, nkv, hd, dtype, fused=B == 5, seed=B + H)
    out, lse = hdf.block_attention_kv4(c.q, c.kv4, 0, **c.kw)
    c.check(out, lse)


@pytest.mark.parametrize("dtype,hd,B,H,nkv", [(BF, 128, 3, 8, 8), (BF, 64, 16, 16, 8), (BF, 128, 5, 56, 8),
                                              (BF, 64, 1, 32, 32), (F32, 128, 2, 16, 8), (F32, 64, 17, 8, 8)])
@pytest.mark.parametrize("long", [130, 700])
def test_many_short_contexts(dtype, hd, B, H, nkv, long):
    """More workgroups than the card has compute units, for which smaller ones are taken."""
    print(f"[kv4 attention] many, hd={hd} {dtype} B={B} H={H}/{nkv} long={long}", flush=True)
    n = 44 if nkv == 8 else 11
    ctx = ([0, 1, 63, 64, 65, 127, 128, 129, long, 2, 100] * 4)[:n]
    c = Case(ctx, B, H, nkv, hd, dtype, seed=20 + B)
    blen = [s % (B + 1) for s in range(n)]
    bl = torch.tensor(blen, dtype=torch.int32, device="cuda")
    out = torch.full_like(c.q, 77.0)
    lse = torch.full((n, B, H), 55.0, device="cuda")
    hdf.block_attention_kv4(c.q, c.kv4, 0, block_len=bl, causal=True, out=(out, lse), **c.kw)
    c.check(out, lse, causal=True, blen=blen)
    for s, b in enumerate(blen):
        assert (out[s, b:] == 77.0).all() and (lse[s, b:] == 55.0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("causal", [False, True])
def test_block_lengths_and_causal_slots(dtype, causal):
    c = Case([65, 3, 0, 200], 7, 4, 2, 128, dtype, paged=False, layers=2, layer=1, seed=3)
    blen = [7, 1, 4, 0]
    bl = torch.tensor(blen, dtype=torch.int32, device="cuda")
    out = torch.full_like(c.q, 77.0)
    lse = torch.full((4, 7, 4), 55.0, device="cuda")
    hdf.block_attention_kv4(c.q, c.kv4, 1, block_len=bl, causal=causal, out=(out, lse), **c.kw)
    c.check(out, lse, causal=causal, blen=blen)
    for s, b in enumerate(blen):        # slots behind a block's length
        assert (out[s, b:] == 77.0).all() and (lse[s, b:] == 55.0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_no_key_at_all(dtype):
    c = Case([0, 70, 0], 3, 2, 1, 64, dtype, block=False, seed=4)
    out, lse = hdf.block_attention_kv4(c.q, c.kv4, 0, **c.kw)
    c.check(out, lse)
    assert not out[0].any() and torch.isneginf(lse[0]).all()
    none, l = hdf.block_attention_kv4(c.q, None, ctx_len=torch.zeros_like(c.kw["ctx_len"]), max_ctx=0)
    assert not none.any() and torch.isneginf(l).all()
    c.ctx, c.k, c.v, c.block = [0, 0, 0], [c.k[0]] * 3, [c.v[0]] * 3, True
    out, lse = hdf.block_attention_kv4(c.q, None, ctx_len=torch.zeros_like(c.kw["ctx_len"]), max_ctx=0,
                                       k_blk=c.kb, v_blk=c.vb)
    c.check(out, lse)


@pytest.mark.parametrize("dtype,ctx", [(BF, [20000]), (F32, [9000]), (BF, [4000, 1, 2500])])
def test_long_contexts_in_pieces(dtype, ctx):
    c = Case(ctx, 2, 4, 2, 128, dtype, seed=5)
    out, lse = hdf.block_attention_kv4(c.q, c.kv4, 0, **c.kw)
    c.check(out, lse)
    again, lse2 = hdf.block_attention_kv4(c.q, c.kv4, 0, **c.kw)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


def test_sharp_scores_and_a_scale():
    """Scores of a few hundred: one key takes nearly all of the weight."""
    c = Case([300, 64], 4, 4, 4, 128, BF, spread=4.0, seed=6)
    out, lse = hdf.block_attention_kv4(c.q, c.kv4, 0, scale=0.7, **c.kw)
    c.check(out, lse, scale=0.7)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("sizes", [(1e30, 1e-30), (1e-27, 1e-30), (2e33, 3e33), (1e-20, 1e20)])
def test_values_of_any_size(dtype, sizes):
    """Values far from 1, and of different sizes in one context: the factor that carries a value's
    scale follows the greatest so far, in either order."""
    c = Case([130, 200], 3, 2, 2, 64, dtype, seed=13, block=False)
    for s, T in enumerate(c.ctx):
        g = torch.Generator().manual_seed(s)
        size = torch.where(torch.rand(T, 1, 1, generator=g) < 0.5, sizes[s], sizes[1 - s])
        v = (torch.randn(T, 2, 64, generator=g) * size).to(dtype)
        pages = c.kw["page_table"][s].tolist()
        hdf.kv4_write_rows(c.kv4, 0, None, v.view(T, -1).cuda(), rows=hdf.paged_rows(pages, T, "cuda"))
        c.v[s] = ref.quantise_values(_np(v))
    out, lse = hdf.block_attention_kv4(c.q, c.kv4, 0, **c.kw)
    c.check(out, lse)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", [1e-30, 1e8, 1e12, 1e30, 1e36])
@pytest.mark.parametrize("ctx", [[0, 40], [700, 130]])
def test_block_values_of_any_size(dtype, size, ctx):
    """Values of the block far from 1, alone and beside a context of ordinary ones."""
    c = Case(ctx, 7, 4, 2, 128, dtype, seed=15)
    c.vb.mul_(size)
    c.vb[1, 3, 1, 5] *= 16
    out, lse = hdf.block_attention_kv4(c.q, c.kv4, 0, **c.kw)
    assert torch.isfinite(out.float()).all()
    c.check(out, lse)


@pytest.mark.parametrize("dtype,hd,B,H", [(BF, 128, 9, 4), (BF, 64, 6, 2), (F32, 128, 9, 2), (F32, 64, 9, 4)])
def test_what_is_no_number_in_masked_slots(dtype, hd, B, H):
    """A causal slot does not see the slots after it, whatever they hold, nor any slot those from
    the block's length on."""
    c = Case([100, 0], B, H, 2, hd, dtype, seed=16)
    blen = [B, 4]
    kw = dict(c.kw, block_len=torch.tensor(blen, dtype=torch.int32, device="cuda"))
    want, lse0 = hdf.block_attention_kv4(c.q, c.kv4, 0, causal=True, **kw)
    nan, inf = float("nan"), float("inf")
    c.vb[0, 5, 0, 3] = nan                # seen from slot 5 on
    c.vb[0, 4, 1, 7], c.vb[0, 5, 1, 7] = inf, -inf
    c.vb[0, 3, 1, 9] = -inf
    c.kb[0, 5, 0, 0] = nan                # the scores of head 0 from slot 5 on
    c.kb[1, 4:], c.vb[1, 4:] = nan, inf
    out, lse = hdf.block_attention_kv4(c.q, c.kv4, 0, causal=True, **kw)
    G = H // 2
    assert torch.equal(out[1, :4], want[1, :4]) and torch.equal(lse[1, :4], lse0[1, :4])
    # A value that is no number moves the power of two that probabilities are taken relative to, and
    # with it the rounding of the exponentials' arguments (2^-18 each side) and of what follows.
    tol = 2.0 ** -7 if dtype == BF else 2.0 ** -16
    near = lambda a, b: torch.allclose(a.float(), b.float(), rtol=tol, atol=tol * float(want.abs().max()))
    assert near(out[0, :5, :G], want[0, :5, :G]) and near(lse[0, :5], lse0[0, :5])
    assert torch.isnan(out[0, 5:, :G]).all() and torch.isnan(lse[0, 5:, :G]).all()
    assert near(lse[0, :, G:], lse0[0, :, G:])
    got, ref_ = out[0, :, G:].clone(), want[0, :, G:].clone()
    assert (got[3:, :, 9] == -inf).all() and (got[4, :, 7] == inf).all() and torch.isnan(got[5:, :, 7]).all()
    got[3:, :, 9] = ref_[3:, :, 9]
    got[4:, :, 7] = ref_[4:, :, 7]
    assert near(got, ref_)


def test_a_cache_beyond_32_bits():
    """Pages at the end of a cache of more than 4 GiB."""
    c = Case([300], 4, 8, 8, 128, BF, seed=14)
    tiles = 66000
    kv4 = torch.zeros((1, 8, tiles, 8576), dtype=torch.uint8, device="cuda")
    assert kv4.numel() > 1 << 32
    n = c.kv4.shape[2]
    kv4[:, :, tiles - n:] = c.kv4
    c.kw["page_table"] = c.kw["page_table"] + (tiles - n)
    out, lse = hdf.block_attention_kv4(c.q, kv4, 0, **c.kw)
    c.check(out, lse)


def test_pages_outside_the_pool_hold_no_keys():
    c = Case([200], 4, 2, 2, 64, BF, seed=7)
    pt = c.kw["page_table"]
    pt[0, 1] = -5
    pt[0, 3] = c.kv4.shape[2]
    keep = np.r_[0:64, 128:192]
    c.k[0], c.v[0] = c.k[0][keep], c.v[0][keep]
    out, lse = hdf.block_attention_kv4(c.q, c.kv4, 0, **c.kw)
    c.check(out, lse)


def test_rows_that_are_no_numbers_reach_their_heads_alone():
    c = Case([100, 50], 2, 4, 2, 64, BF, seed=8)
    bad = torch.zeros(1, 2 * 64, dtype=BF, device="cuda")
    bad[0, 70] = float("nan")           # of head 1
    page = int(c.kw["page_table"][0, 1])
    hdf.kv4_write_rows(c.kv4, 0, bad, None, row0=64 * page + 5)
    out, lse = hdf.block_attention_kv4(c.q, c.kv4, 0, **c.kw)
    assert torch.isnan(out[0, :, 2:]).all() and torch.isnan(lse[0, :, 2:]).all()
    assert torch.isfinite(out[0, :, :2]).all() and torch.isfinite(out[1]).all()


def test_a_larger_workspace_serves_and_lse_is_optional():
    c = Case([3000, 10], 3, 4, 2, 128, BF, seed=9)
    need = hdf.block_attention_kv4_workspace(2, 3, 4, 2, 128, 9000)
    ws = torch.full((need + 512,), 0xFF, dtype=torch.uint8, device="cuda")
    want, _ = hdf.block_attention_kv4(c.q, c.kv4, 0, **c.kw)
    got, lse = hdf.block_attention_kv4(c.q, c.kv4, 0, want_lse=False, ws=ws, **c.kw)
    assert lse is None and torch.equal(want, got)


def test_written_and_attended_to_in_a_graph():
    """A round (new rows into the cache, then the block) captured and replayed, with eager work and
    other contents between the replays."""
    c = Case([700, 3000], 4, 4, 2, 128, BF, seed=10)
    nkv, hd = c.nkv, c.hd
    rows = torch.cat([hdf.paged_rows(c.kw["page_table"][s].tolist(), t, "cuda")[-3:]
                      for s, t in enumerate(c.ctx)]).contiguous()
    k = torch.zeros(6, nkv * hd, dtype=BF, device="cuda")
    v = torch.zeros_like(k)
    out = (torch.zeros_like(c.q), torch.zeros(2, 4, 4, device="cuda"))
    ws = torch.zeros(hdf.block_attention_kv4_workspace(2, 4, 4, nkv, hd, c.max_ctx), dtype=torch.uint8,
                     device="cuda")

    def step(o):
        hdf.kv4_write_rows(c.kv4, 0, k, v, rows=rows)
        hdf.block_attention_kv4(c.q, c.kv4, 0, out=o, ws=ws, **c.kw)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(out)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out)
    for i in range(4):
        g = torch.Generator(device="cuda").manual_seed(i)
        k.copy_(torch.randn(k.shape, generator=g, device="cuda"))
        v.copy_(torch.randn(v.shape, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in out]
        want = (torch.zeros_like(c.q), torch.zeros_like(out[1]))
        step(want)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i


def test_two_streams_at_once():
    a, b = Case([2500], 4, 4, 4, 64, BF, seed=11), Case([90, 4000], 2, 8, 2, 128, F32, seed=12)
    torch.cuda.synchronize()
    sides = torch.cuda.Stream(), torch.cuda.Stream()
    got = [hdf.block_attention_kv4(c.q, c.kv4, 0, stream=s, **c.kw)
           for _ in range(5) for c, s in zip((a, b), sides)][-2:]
    for s in sides:
        s.synchronize()
    a.check(*got[0])
    b.check(*got[1])
