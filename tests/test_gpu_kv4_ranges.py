"""GPU tests of hdf_block_attention_kv4 where values of very different sizes, infinities or NaN stand
beside ordinary ones: what a query gives no weight, or does not see, leaves its output's precision as
it is.

Bound of an output element, with A = sum p |v| over the keys that are seen, and W the greatest p |v|
of a key's whole head:
  a score is off by d <= (hd + 6) 2^-24 scale sum |q k| + 2^-22 (fp32 sums of hd products and the two
  roundings of the exponential's argument; the exponential), its probability by a factor 1 + d, the
  ratio of sums by 2 d; bf16: a context probability times its value's scale is rounded to fp16, 2^-11
  of itself, or half a step of fp16's subnormals, 2^-23 of the greatest probability times that key's
  scale (which is at most |v| / 6 of its head), or is two bf16 terms, 2^-16 of itself; fp32: a
  probability in three bf16 terms, 2^-24, a query in three, 2^-24 more of its score; sums over N keys
  in fp32, each at most N 2^-24, of outputs and of weights; the result is rounded once, 2^-8 of itself
  (bf16) or 2^-24 (fp32).  Below fp32's least normal number may be 0: a probability relative to the
  greatest and the lower term it is split into, 2 * 2^-126 max |v| a key; a sum in its unit, which is
  2^-86 beside values of 2^40 and more.
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
    """Contexts in slots of their own, values of about `size`, a block, queries of noise."""

    def __init__(self, ctx, B, H, nkv, hd, dtype, size, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        noise = lambda *shape: torch.randn(shape, generator=g, device="cuda")
        n = len(ctx)
        self.ctx, self.B, self.H, self.nkv, self.hd, self.dtype = ctx, B, H, nkv, hd, dtype
        self.offs = hdf.kv_slot_offsets(ctx)
        self.kv4 = hdf.kv4_alloc(1, nkv, hd, self.offs[-1] + 64)
        self.kv4.fill_(0xFF)            # rows that no sequence holds: NaN scales
        for s, T in enumerate(ctx):
            if T:
                self.put(s, 0, noise(T, nkv, hd), noise(T, nkv, hd) * size)
        self.q = noise(n, B, H, hd).to(dtype)
        self.kb, self.vb = noise(n, B, nkv, hd).to(dtype), (noise(n, B, nkv, hd) * size).to(dtype)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.kw = dict(ctx_len=torch.tensor(ctx, **i32), max_ctx=max(ctx), k_blk=self.kb, v_blk=self.vb,
                       kv_offsets=torch.tensor(self.offs, **i32))

    def put(self, s, at, k, v):
        """Rows `at` .. of sequence s."""
        flat = [None if x is None else x.to(self.dtype).reshape(x.shape[0], -1).contiguous().cuda()
                for x in (k, v)]
        hdf.kv4_write_rows(self.kv4, 0, *flat, row0=self.offs[s] + at)

    def rows(self, s):
        """What the cache stands for; codes times scales are exact in 32 bits."""
        T = self.ctx[s]
        k, v = hdf.kv4_read_rows(self.kv4, 0, T, row0=self.offs[s], dtype=F32)
        return [_np(x.view(T, self.nkv, self.hd)) for x in (k, v)]

    def __call__(self, causal=False):
        return hdf.block_attention_kv4(self.q, self.kv4, 0, causal=causal, **self.kw)


def _check(c, out, lse, *, causal=False, slots=None):
    """Slots slots[s] (all) of every sequence against the oracle."""
    f32 = c.dtype == F32
    for s, T in enumerate(c.ctx):
        B = c.B if slots is None else slots[s]
        ks, vs = c.rows(s)
        kb, vb, q = _np(c.kb[s, :B]), _np(c.vb[s, :B]), _np(c.q[s, :B])
        o, l, mass, reach = ref.attend(q, ks, vs, kb, vb, causal=causal)
        G, scale = c.H // c.nkv, c.hd ** -0.5
        W, top = np.zeros((B, c.H)), np.zeros((B, c.H))
        for b in range(B):
            for h in range(c.H):
                p = np.exp(scale * (ks[:, h // G] @ q[b, h]) - l[b, h])
                heads = np.abs(vs[:, h // G]).max(1, initial=0.0)
                n = b + 1 if causal else B
                W[b, h] = (p * heads).max(initial=0.0)
                top[b, h] = max(heads.max(initial=0.0), np.abs(vb[:n, h // G]).max())
        d = (c.hd + 6) * 2.0 ** -24 * reach + 2.0 ** -22 + (2.0 ** -24 * reach if f32 else 0.0)
        N = T + B
        tol = mass * (2 * d[..., None] + (2.0 ** -24 if f32 else 2.0 ** -11) + 2 * N * 2.0 ** -24)
        tol += np.abs(o) * (2.0 ** -24 if f32 else 2.0 ** -8)
        least = 2 * 2.0 ** -126 * top + np.where(top >= 2.0 ** 40, 6 * 2.0 ** -86, 6 * 2.0 ** -126)
        tol += N * (least + (0.0 if f32 else 2.0 ** -23 * W))[..., None]
        err = np.abs(_np(out[s, :B]) - o)
        worst = float((err / np.maximum(mass, 1e-300)).max(initial=0.0))
        assert (err <= tol).all(), (s, T, worst, np.argwhere(~(err <= tol))[:3])
        e = np.abs(_np(lse[s, :B]) - l)
        bound = d + N * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(l))
        assert (e <= bound).all(), (s, T, float((e - bound).max()))


FORMS = [(BF, 128, 9, 4), (BF, 64, 6, 2), (BF, 128, 9, 8), (F32, 128, 9, 2), (F32, 64, 9, 4)]


@pytest.mark.parametrize("dtype,hd,B,H", FORMS)
@pytest.mark.parametrize("size", [1.0, 0.02, 1e-3])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 3e38, 2.0 ** 70])
def test_unseen_slots_leave_the_others_as_they_are(dtype, hd, B, H, size, bad):
    """Contexts of 10 to 63 tiles under a causal block whose later slots hold what is no number, or
    nearly none; a dim of a slot that sees it keeps its precision in the others."""
    print(f"[kv4 ranges] unseen {dtype} hd={hd} B={B} H={H} size={size} bad={bad}", flush=True)
    c = Case([1030, 600, 4000, 0], B, H, 2, hd, dtype, size, 41)
    clean, lse0 = c(causal=True)
    c.vb[:, 5:, :, 3] = bad
    out, lse = c(causal=True)
    _check(c, out, lse, causal=True, slots=[5] * 4)
    assert torch.equal(out[:, :5], clean[:, :5]) and torch.equal(lse, lse0)
    others = [d for d in range(hd) if d != 3]
    assert torch.equal(out[..., others], clean[..., others])


@pytest.mark.parametrize("dtype,hd,B,H", FORMS)
@pytest.mark.parametrize("big", [2.0 ** 14, 2.0 ** 26, 1e10, 2.0 ** 40, 1e20, 1e30])
@pytest.mark.parametrize("where", ["first", "middle", "last"])
def test_a_row_of_large_values_and_no_weight(dtype, hd, B, H, big, where):
    """Ordinary rows beside one whose values are far larger and whose probability is 2^-100 or so."""
    print(f"[kv4 ranges] large {dtype} hd={hd} B={B} H={H} big={big} {where}", flush=True)
    c = Case([700, 1500, 4000], B, H, 2, hd, dtype, 0.02, 42)
    c.q[..., 0] = 8.0
    for s, T in enumerate(c.ctx):
        k, v = torch.zeros(1, 2, hd), torch.randn(1, 2, hd, generator=torch.Generator().manual_seed(7))
        k[0, :, 0] = -8.75 * hd ** 0.5           # a score of -70, about 2^-100
        c.put(s, {"first": 1, "middle": T // 2, "last": T - 2}[where], k, v * big)
    out, lse = c()
    _check(c, out, lse)


@pytest.mark.parametrize("dtype,hd,B,H", FORMS)
@pytest.mark.parametrize("small", [0.0, 1e-30, 2.0 ** -30, 2.0 ** -14])
@pytest.mark.parametrize("where", ["first", "last", "block"])
def test_a_row_of_small_values_and_all_the_weight(dtype, hd, B, H, small, where):
    """Rows of about 2^-40 of the weight beside one that has the rest and the smallest values, in the
    context or in the block: the output is of the size of either part's."""
    print(f"[kv4 ranges] small {dtype} hd={hd} B={B} H={H} small={small} {where}", flush=True)
    c = Case([700, 1500, 4000], B, H, 2, hd, dtype, 1.0, 43)
    c.q[..., 0] = 8.0
    k, v = torch.zeros(1, 2, hd), torch.randn(1, 2, hd, generator=torch.Generator().manual_seed(8)) * small
    k[0, :, 0] = 3.5 * hd ** 0.5                 # a score of 28, about 2^40
    if where == "block":
        c.kb[:, 2:3], c.vb[:, 2:3] = k.to(c.dtype).cuda(), v.to(c.dtype).cuda()
    else:
        for s, T in enumerate(c.ctx):
            c.put(s, 3 if where == "first" else T - 3, k, v)
    out, lse = c()
    _check(c, out, lse)


@pytest.mark.parametrize("dtype,hd,B,H", FORMS)
@pytest.mark.parametrize("spread", [1.0, 4.0, 10.0])
def test_values_of_sizes_that_vary(dtype, hd, B, H, spread):
    """Sizes of rows from a log-normal distribution: a factor of 2 either way to one of 2^10."""
    print(f"[kv4 ranges] spread {dtype} hd={hd} B={B} H={H} spread={spread}", flush=True)
    c = Case([700, 1500, 4000], B, H, 2, hd, dtype, 1.0, 44)
    for s, T in enumerate(c.ctx):
        g = torch.Generator().manual_seed(s)
        size = torch.exp2(spread * torch.randn(T, 2, 1, generator=g))
        c.put(s, 0, None, torch.randn(T, 2, hd, generator=g) * size)
    out, lse = c()
    _check(c, out, lse)


@pytest.mark.parametrize("dtype,hd", [(BF, 64), (BF, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("size", [1e30, 1e36, 5e37])
def test_sums_of_large_values(dtype, hd, size):
    """Many keys of nearly the same score whose values' sum is beyond the type while their mean is
    not, in the context and in the block."""
    print(f"[kv4 ranges] sums {dtype} hd={hd} size={size}", flush=True)
    c = Case([4096, 300, 0], 64, 2, 1, hd, dtype, 1.0, 45)
    for s, T in enumerate(c.ctx):
        if T:
            g = torch.Generator().manual_seed(s)
            c.put(s, 0, None, torch.rand(T, 1, hd, generator=g) * size)
    c.vb.copy_(torch.rand(c.vb.shape, generator=torch.Generator().manual_seed(9)) * size)
    c.q.mul_(0.01)
    out, lse = c()
    assert torch.isfinite(out.float()).all()
    _check(c, out, lse)


@pytest.mark.parametrize("dtype,hd", [(BF, 128), (F32, 64)])
@pytest.mark.parametrize("ctx", [700, 5000])
def test_log_sum_exp_of_equal_scores(dtype, hd, ctx):
    """Queries of zeros: the sum is the number of keys, exactly, and its logarithm off by the
    logarithm's last place and a product's rounding, whatever the values are."""
    c = Case([ctx], 4, 2, 1, hd, dtype, 1e-28, 46)
    c.q.zero_()
    out, lse = c()
    want = np.log(ctx + 4.0)
    assert (np.abs(_np(lse) - want) <= 2.0 ** -22 * (1 + want)).all()
    _check(c, out, lse)


@pytest.mark.parametrize("dtype,hd,B,H", [(BF, 128, 3, 8), (BF, 128, 9, 16), (BF, 64, 16, 16), (F32, 64, 9, 16)])
def test_many_short_contexts_of_sizes_that_vary(dtype, hd, B, H):
    """More workgroups than the card has compute units, for which smaller ones are taken: sizes of a
    factor of 2^10 either way, causal, NaN in the last slot."""
    print(f"[kv4 ranges] many {dtype} hd={hd} B={B} H={H}", flush=True)
    c = Case(([0, 1, 64, 65, 130, 300, 513, 700] * 5)[:36], B, H, 8, hd, dtype, 1.0, 47)
    for s, T in enumerate(c.ctx):
        if T:
            g = torch.Generator().manual_seed(s)
            size = torch.exp2(10 * torch.randn(T, 8, 1, generator=g))
            c.put(s, 0, None, torch.randn(T, 8, hd, generator=g) * size)
    c.vb[:, B - 1] = float("nan")
    out, lse = c(causal=True)
    _check(c, out, lse, causal=True, slots=[B - 1] * len(c.ctx))
    assert torch.isnan(out[:, B - 1]).all()


@pytest.mark.parametrize("place", ["first", "last", "all"])
def test_a_chunk_of_as_many_tiles_as_a_workgroup_takes(place):
    """32768 positions in one chunk, 64 tiles a wave: large values without weight in the first or the
    last tile of a wave, or in every second one."""
    c = Case([32768] + [0] * 32, 1, 8, 8, 64, BF, 0.02, 48)
    c.q[..., 0] = 8.0
    k, v = torch.zeros(1, 8, 64), torch.randn(1, 8, 64, generator=torch.Generator().manual_seed(7)) * 1e10
    k[0, :, 0] = -8.75 * 8                       # a score of -70
    for t in {"first": [0], "last": [511], "all": range(0, 512, 2)}[place]:
        c.put(0, 64 * t + 63, k, v)
    out, lse = c()
    _check(c, out, lse)
