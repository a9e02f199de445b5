"""Truncated draws, their verification and top logits on the GPU against the float64 oracle.

Draws, cuts and identities are whole numbers and have to be equal: both sides sum in 64 bits, and
no row is built so that a cut falls within 1e-9 of a border unless its sums are exact.  The
log-sum-exps are 64-bit: the kernels' exponentials drop less than 1e-14 of a term and the sums
of V terms round by V * 2^-53 at most, so 1e-10 relative to max(1, |lse|) covers 2^17 columns."""
import math

import numpy as np
import pytest
import torch

from oracle import truncation as tr
from paper_2606_26744_amd import hdf

pytestmark = pytest.mark.gpu
DEV = "cuda"
LSE_TOL = 1e-10


def _logits(rows, V, seed, dtype=torch.float32, kind="peaked", ld=None, offset=0):
    """[rows, V] device logits with row stride ld whose first element lies `offset` elements into
    the allocation."""
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(rows, V, generator=g) * (1.3 if kind == "flat" else 1.8)
    if kind == "peaked":
        head = torch.randint(0, V, (rows, 48), generator=g)
        z.scatter_reduce_(1, head, torch.rand(rows, 48, generator=g) * 9 + 5, "amax")
    if kind == "ties":
        z = (z * 2).round() / 2
    ld = ld or V
    buf = torch.full((rows * ld + offset + 8,), 77.0, dtype=dtype, device=DEV)
    out = torch.as_strided(buf, (rows, V), (ld, 1), offset)
    out.copy_(z)
    return out


def _np(t):
    return t.detach().cpu().double().numpy()


def _value(x, r, per):
    return x if not torch.is_tensor(x) else x[r // per].item()


def _check_draws(z, u=None, per=1, rows=None, **kw):
    """rows: those to compare (all)."""
    tok, cut = hdf.sample_truncated(z, u, rows_per_seq=per, **kw)
    torch.cuda.synchronize()
    for r in range(z.shape[0]) if rows is None else rows:
        s = {k: _value(v, r, per) for k, v in kw.items()}
        n, cl, ci, lse, p = tr.truncate(_np(z[r]), **s)
        assert int(cut.kept[r]) == n, (r, s)
        assert float(cut.cut_logit[r]) == cl and int(cut.cut_index[r]) == ci, (r, s)
        got = float(cut.lse[r])
        assert got == lse or abs(got - lse) <= LSE_TOL * max(1.0, abs(lse)), (r, got, lse)
        if u is not None:
            assert int(tok[r]) == tr.inverse(p, float(u[r])), (r, s)
    return tok, cut


def _u(rows, seed):
    return torch.rand(rows, generator=torch.Generator().manual_seed(seed)).to(DEV)


SETTINGS = {
    "open": dict(),
    "top_k": dict(temperature=0.8, top_k=50),
    "top_p": dict(top_p=0.95),
    "warm": dict(temperature=1.5, top_p=0.95),
    "min_p": dict(temperature=0.7, min_p=0.05),
    "all": dict(temperature=0.9, top_k=40, top_p=0.9, min_p=0.02),
    "greedy": dict(temperature=0.0, top_p=0.5),
    "one": dict(top_k=1),
    "first": dict(top_p=0.0),
    "equals": dict(min_p=1.0),
    "hot": dict(temperature=50.0, top_p=0.5),
    "cold": dict(temperature=1e-3, top_p=0.9),
    "wide_k": dict(top_k=3000, top_p=0.99),
}


@pytest.mark.parametrize("name", list(SETTINGS))
@pytest.mark.parametrize("kind", ["peaked", "flat", "ties"])
def test_draws_every_setting(name, kind):
    z = _logits(5, 8191, 11, kind=kind, ld=8200)
    _check_draws(z, _u(5, 3), **SETTINGS[name])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 63, 257, 1024, 4095, 4097, 12289, 32003])
def test_draws_every_length(V, dtype):
    z = _logits(3, V, V, dtype, kind="peaked" if V > 100 else "flat", ld=V + 3, offset=1)
    for kw in (dict(), dict(top_k=5), dict(top_p=0.8), dict(top_k=700, top_p=0.95, min_p=1e-4)):
        _check_draws(z, _u(3, V), **kw)


@pytest.mark.parametrize("V,dtype,kind,name", [
    (129280, torch.float32, "peaked", "all"), (129280, torch.bfloat16, "flat", "warm"),
    (151937, torch.float32, "flat", "top_p"), (1 << 20, torch.float32, "flat", "open"),
    (1 << 20, torch.bfloat16, "flat", "warm"), ((1 << 20) - 1, torch.float32, "peaked", "top_k")])
def test_draws_long_rows(V, dtype, kind, name):
    _check_draws(_logits(2, V, 5, dtype, kind, ld=V + 1), _u(2, 9), **SETTINGS[name])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", range(0, 9))
def test_draws_every_alignment(offset, dtype):
    z = _logits(4, 5003, offset, dtype, ld=5005, offset=offset)
    before = z.clone()
    _check_draws(z, _u(4, offset), top_p=0.9)
    assert torch.equal(z, before)


def test_settings_per_sequence():
    """An entry a sequence, odd values among them: greedy by 0, by a negative and a NaN
    temperature, filters off by every documented value, a last sequence of fewer rows."""
    nan = float("nan")
    T = torch.tensor([0.0, -1.0, 0.7, 1.0, 1.3, 2.0], device=DEV)
    k = torch.tensor([0, 5, -3, 1 << 30, 17, 2], dtype=torch.int32, device=DEV)
    p = torch.tensor([0.9, 1.0, 2.0, 0.5, -1.0, 0.99], device=DEV)
    m = torch.tensor([0.0, 0.1, -0.5, 0.01, 1.5, 0.0], device=DEV)
    z = _logits(22, 9001, 3)
    _check_draws(z, _u(22, 4), per=4, temperature=T, top_k=k, top_p=p, min_p=m)
    T2 = torch.tensor([nan], device=DEV)
    tok, cut = hdf.sample_truncated(z[:1], _u(1, 1), temperature=T2,
                                    top_p=torch.tensor([nan], device=DEV),
                                    min_p=torch.tensor([nan], device=DEV))
    assert int(cut.kept[0]) == 1 and int(tok[0]) == int(z[0].argmax())
    off = torch.tensor([nan], device=DEV)
    tok, cut = hdf.sample_truncated(z[:1], _u(1, 1), top_p=off, min_p=off)
    assert int(cut.kept[0]) == 9001


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masked_rows(dtype):
    """-inf and NaN in masked places, the type's lowest value as a mask, rows with one entry and
    with none, masks that cover whole stretches."""
    V = 20011
    z = _logits(9, V, 21, dtype)
    z[0] = -np.inf
    z[1] = -np.inf
    z[1, 13007] = -4.0
    z[2, ::3] = float("nan")
    z[3] = torch.finfo(dtype).min
    z[4, 100:] = torch.finfo(dtype).min
    z[5, :19000] = -np.inf
    z[6, 7:] = -np.inf
    z[7] = float("nan")
    z[8, torch.randperm(V)[:V - 300].to(DEV)] = -np.inf
    for kw in (dict(), dict(top_k=50), dict(top_p=0.9), dict(top_k=700), dict(min_p=0.01),
               dict(temperature=0.3, top_k=200, top_p=0.95), dict(temperature=0.0)):
        _check_draws(z, _u(9, 8), **kw)


def test_many_equal_entries():
    """Whole rows of one value, two values, values a few ulps or denormals apart: cuts fall among
    thousands of ties, in token order.  The sums are exact or far from the borders."""
    V = 70001
    z = torch.zeros(6, V, device=DEV)
    z[1, ::2] = -1.0
    z[2] = torch.randint(0, 3, (V,), generator=torch.Generator().manual_seed(1)).float().to(DEV)
    z[3] = 7 + torch.arange(V, device=DEV).remainder(5) * 2.0 ** -21
    z[4] = torch.arange(V, device=DEV).remainder(911) * 1.4e-45
    z[5, 1::2] = -0.0
    for kw in (dict(), dict(top_p=0.5), dict(top_k=30001), dict(top_k=1), dict(min_p=1.0),
               dict(top_k=50000, top_p=0.25), dict(temperature=1e-4, top_p=0.7)):
        _check_draws(z, _u(6, 2), **kw)


@pytest.mark.parametrize("V", [2, 56, 640, 4096, 8192, 32768, 131072])
@pytest.mark.parametrize("n", [3, 258])
def test_equal_entries_on_the_border(n, V):
    """Rows of equal logits, alone, above ones that weigh nothing and among masked ones: a nucleus of
    a dyadic share holds exactly that many, and a uniform on the border between two tokens takes the
    second: n weights of one sum to n."""
    z = torch.full((n, V), 3.7, device=DEV)
    z[1, V // 2:] = -1e4
    z[2, ::2] = -np.inf
    z[2] -= 90.3
    live = [np.arange(V), np.arange(V // 2), np.arange(1, V, 2)]   # the equal ones, as columns
    for dtype in (torch.float32, torch.bfloat16):
        x = z.to(dtype)
        for T in (1.0, 0.7):
            for kw in (dict(top_p=0.5), dict(top_p=0.25), dict(top_p=0.75), dict(min_p=1.0),
                       dict(top_k=max(1, V // 4), top_p=0.5)):
                for at in (0.5, 0.25, 3 / 128):
                    tok, cut = hdf.sample_truncated(x, torch.full((n,), at, device=DEV), temperature=T,
                                                    **kw)
                    for r, cols in enumerate(live):
                        # n weights of one sum to n: the first to pass u n is number floor(u n).
                        most = min(len(cols), kw.get("top_k", V))
                        want = math.ceil(most * kw.get("top_p", 1.0))
                        assert int(cut.kept[r]) == want, (r, kw)
                        assert int(tok[r]) == cols[math.floor(at * want)], (r, kw, at)
                        every = want == (len(cols) if r != 1 else V)
                        assert int(cut.cut_index[r]) == (-1 if every else cols[want - 1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_nuclei_wider_than_the_lists(dtype):
    """Thousands of kept entries, cuts in bins of a few and of thousands of entries, with and without
    min_p above or below them."""
    z = _logits(3, 200003, 41, dtype, "flat")
    z[2, :150000] = -np.inf
    for kw in (dict(temperature=1.5, top_p=0.5), dict(temperature=3.0, top_p=0.9),
               dict(temperature=1.0, top_p=0.999), dict(temperature=30.0, top_p=0.3),
               dict(top_p=0.9, min_p=0.001), dict(top_p=0.9, min_p=0.02), dict(min_p=0.01),
               dict(top_k=70000, top_p=0.6), dict(top_k=5000, min_p=0.03)):
        _check_draws(z, _u(3, 5), **kw)


def test_many_rows():
    """More rows than one launch of large workgroups takes: lists in small ones, the rest after."""
    n, V = 300, 6007
    z = _logits(n, V, 17)
    z[100:200] = _logits(100, V, 18, kind="flat")
    z[7] = -np.inf
    z[8] = 1.0
    g = torch.Generator().manual_seed(3)

    def pick(values, dtype):
        return torch.tensor(values, dtype=dtype)[torch.randint(0, len(values), (n // 3,), generator=g)
                                                 ].to(DEV)
    _check_draws(z, _u(n, 2), per=3, temperature=pick([0.0, 0.7, 1.0, 1.5], torch.float32),
                 top_k=pick([0, 0, 10, 200, 4000], torch.int32),
                 top_p=pick([1.0, 0.9, 0.99, 0.5], torch.float32),
                 min_p=pick([0.0, 0.0, 0.05], torch.float32))
    _check_draws(z, None, top_p=0.8)
    ids, values, rest = hdf.top_logits(z, 40)
    for r in range(n):
        i, v, s = tr.top_logits(_np(z[r]), 40)
        assert ids[r].tolist() == i.tolist() and _np(values[r]).tolist() == v.tolist(), r
        assert float(rest[r]) == s or abs(float(rest[r]) - s) <= 2e-7 * max(1.0, abs(s)), r


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [3, 259])
def test_borders_of_many_entries(n, dtype):
    """A nucleus' border falls among a few, some thousand (more than a row's lists hold) and more
    entries than are held at once, of distinct values and of ties, in few rows and in many."""
    V = 60013
    z = _logits(n, V, 51, dtype, "flat")
    z[1] = (z[1] * 4).round() / 4
    rows = (0, 1, n - 1)
    for kw in (dict(temperature=1.5, top_p=0.95), dict(temperature=3.0, top_p=0.5),
               dict(temperature=12.0, top_p=0.7), dict(temperature=3.0, min_p=0.4),
               dict(temperature=3.0, top_p=0.6, min_p=0.37), dict(top_p=0.999, min_p=1e-6)):
        _check_draws(z, _u(n, 12), rows=rows, **kw)


@pytest.mark.parametrize("n", [2, 258])
def test_weights_far_below_the_greatest(n):
    """Entries many octaves below a row's greatest: kept by a tiny min_p, weightless in a draw;
    temperatures so low that any other entry weighs nothing; a greatest value of zero, of the least
    and of the greatest magnitude."""
    V = 9001
    z = _logits(n, V, 61, kind="flat")
    rows = (0, 1, n - 1)
    for kw in (dict(temperature=0.05, min_p=1e-20), dict(temperature=0.05, min_p=1e-17),
               dict(temperature=0.05, top_p=0.999999), dict(temperature=0.02),
               dict(temperature=0.03, min_p=1e-38, top_p=0.9)):
        _check_draws(z, _u(n, 3), rows=rows, **kw)
    top = z - z.max(1, keepdim=True).values
    for T in (1e-42, 1e-38, 1e-30):
        for kw in (dict(top_p=0.9), dict(), dict(min_p=0.5), dict(top_k=3)):
            _check_draws(top, _u(n, 4), rows=rows, temperature=T, **kw)
    for scale in (1e-38, 1e30):
        for kw in (dict(top_p=0.9), dict(), dict(min_p=0.5)):
            _check_draws(z * scale, _u(n, 5), rows=rows, temperature=scale, **kw)
    inf = torch.full((n,), float("inf"), device=DEV)
    _, cut = hdf.sample_truncated(z, _u(n, 6), temperature=inf, min_p=1.0)
    assert (cut.kept == V).all()   # all weigh the same


def test_rows_in_several_groups_of_launches():
    """So many long rows that they run in turns over one workspace."""
    V, n = 1 << 20, 131
    z = torch.randn(n, V, generator=torch.Generator(DEV).manual_seed(3), device=DEV,
                    dtype=torch.float32).mul_(2).to(torch.bfloat16)
    rows = (0, 1, 125, 126, 127, 130)
    _check_draws(z, _u(n, 1), rows=rows, temperature=0.8, top_p=0.7)
    _check_draws(z, _u(n, 2), rows=rows, top_k=30)
    ids, values, _ = hdf.top_logits(z, 17)
    for r in rows:
        i, v, _ = tr.top_logits(_np(z[r]), 17)
        assert ids[r].tolist() == i.tolist()


def test_rows_more_than_32_bits_apart():
    """Rows whose offsets in elements pass 2^32."""
    V, ld = 5003, 3 * 2 ** 30 + 1
    buf = torch.empty(2 * ld + V, dtype=torch.bfloat16, device=DEV)
    z = torch.as_strided(buf, (3, V), (ld, 1))
    z.copy_(_logits(3, V, 9, torch.bfloat16))
    for kw in (dict(top_p=0.9), dict(top_k=30), dict(temperature=3.0, top_p=0.9), dict()):
        _check_draws(z, _u(3, 1), **kw)
    _check_top(z, 20)


def test_uniforms_at_and_past_the_ends():
    z = _logits(1, 5000, 2).repeat(6, 1)
    u = torch.tensor([0.0, 1 - 2.0 ** -24, 1.0, 7.0, -3.0, float("nan")], device=DEV)
    want = torch.tensor([0.0, 1 - 2.0 ** -24, 1.0, 1.0, 0.0, 0.0])
    for kw in (dict(), dict(top_k=20), dict(top_p=0.8)):
        tok, _ = hdf.sample_truncated(z, u, **kw)
        p = tr.truncate(_np(z)[0], **kw)[4]
        assert tok.tolist() == [tr.inverse(p, float(x)) for x in want]


def test_no_draws_and_empty_batches():
    z = _logits(3, 999, 1)
    tok, cut = hdf.sample_truncated(z, top_k=7)
    assert tok is None and cut.kept.tolist() == [7, 7, 7]
    tok, cut = hdf.sample_truncated(z[:0], _u(0, 1), top_k=7)
    assert tok.shape == (0,) and cut.lse.shape == (0,)
    ids, values, rest = hdf.top_logits(z[:0], 4)
    assert ids.shape == (0, 4) and rest.shape == (0,)


# --------------------------------------------------------------------------- top logits

def _check_top(z, K, T=1.0):
    ids, values, rest = hdf.top_logits(z, K, temperature=T)
    torch.cuda.synchronize()
    zn = _np(z)
    for r in range(z.shape[0]):
        i, v, s = tr.top_logits(zn[r], K, T)
        assert ids[r].tolist() == i.tolist(), r
        assert _np(values[r]).tolist() == v.tolist(), r
        got = float(rest[r])
        # rounded once to fp32 from a 64-bit (or, of small summands, nearly so) value
        assert got == s or abs(got - s) <= 2e-7 * max(1.0, abs(s)), (r, got, s)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,K", [(1, 1), (5, 8), (64, 64), (1000, 1000), (1024, 1024), (4097, 3),
                                 (8191, 128), (32003, 20), (32003, 1024), (129280, 256)])
def test_top_logits(V, K, dtype):
    z = _logits(4, V, V + K, dtype, "peaked" if V > 100 else "flat", ld=V + 5, offset=3)
    _check_top(z, K, 1.0)
    _check_top(z, K, 3.0)


def test_top_logits_of_masked_and_equal_rows():
    V = 30007
    z = _logits(7, V, 4)
    z[0] = -np.inf
    z[1] = 2.5
    z[2] = torch.finfo(torch.float32).min
    z[3, 10:] = -np.inf
    z[4, 15000:] = torch.finfo(torch.float32).min
    z[5] = (z[5] * 2).round()
    z[6, ::2] = float("nan")
    for K in (1, 10, 11, 500):
        _check_top(z, K)


def test_top_logits_without_rest():
    z = _logits(2, 3000, 9)
    ids, values, rest = hdf.top_logits(z, 12, want_rest=False)
    assert rest is None
    assert ids[1].tolist() == tr.top_logits(_np(z)[1], 12)[0].tolist()


# ------------------------------------------------------------------------- verification

def _verify_case(n, B, V, seed, dd=torch.float32, td=torch.float32, kind="peaked", near=0.6, **kw):
    z = _logits(n * B, V, seed, dd, kind)
    g = torch.Generator().manual_seed(seed + 1)
    t = torch.randn(n, B, V, generator=g) * near
    t[:, :B - 1] += z.float().cpu().view(n, B, V)[:, 1:]
    t[:, B - 1] += z.float().cpu().view(n, B, V)[:, 0]
    t = t.to(td).to(DEV)
    tok, cut = hdf.sample_truncated(z, _u(n * B, seed + 2), rows_per_seq=B, **kw)
    u = torch.rand(n, B, generator=g).to(DEV)
    return z, t, tok, cut, u


def _check_verify(n, B, V, z, t, tok, cut, u, kw):
    toks0 = torch.full((n * B + 3,), -9, dtype=torch.int32, device=DEV)
    out = tuple(torch.empty(m, dtype=torch.int32, device=DEV) for m in (n, n, n + 1)) + (toks0,)
    res = hdf.accept_truncated(tok[1:], z[1:], tuple(x[1:] for x in cut), t, u, K=B - 1,
                               draft_stride=B, out=out, **kw)
    acc, anc, offs, toks = (x.tolist() for x in res)
    zn, tn = _np(z), _np(t)
    want_offs, want = [0], []
    for s in range(n):
        sk = {k: _value(v, s, 1) for k, v in kw.items()}
        q = np.array([tr.truncate(zn[s * B + 1 + i], **sk)[4] for i in range(B - 1)])
        p = np.array([tr.truncate(tn[s, i], **sk)[4] for i in range(B)])
        k, nxt, commit = tr.accept(tok[s * B + 1:(s + 1) * B].tolist(), q, p, u[s].tolist())
        assert (acc[s], anc[s]) == (k, nxt), s
        want += commit
        want_offs.append(len(want))
    assert offs == want_offs
    assert toks[:len(want)] == want
    assert all(x == -9 for x in toks[len(want):])   # nothing behind the last sequence
    return acc


@pytest.mark.parametrize("dd,td", [(torch.float32, torch.float32), (torch.float32, torch.bfloat16),
                                   (torch.bfloat16, torch.float32),
                                   (torch.bfloat16, torch.bfloat16)])
@pytest.mark.parametrize("name", ["open", "top_k", "top_p", "min_p", "all", "greedy"])
def test_verify(name, dd, td):
    kw = SETTINGS[name]
    case = _verify_case(6, 8, 3001, 31, dd, td, **kw)
    acc = _check_verify(6, 8, 3001, *case, kw)
    assert len(set(acc)) > 1


@pytest.mark.parametrize("n,B,V", [(1, 1, 50), (3, 1, 2000), (2, 2, 1), (2, 2, 5), (1, 16, 32003),
                                   (5, 7, 4097), (2, 70, 500), (1, 3, 151937)])
def test_verify_sizes(n, B, V):
    kw = dict(top_p=0.9)
    _check_verify(n, B, V, *_verify_case(n, B, V, 3 * V + B, kind="flat", **kw), kw)


def test_verify_settings_per_sequence():
    n, B = 6, 4
    kw = dict(temperature=torch.tensor([0.0, 1.0, 0.7, 1.4, 1.0, 0.9], device=DEV),
              top_k=torch.tensor([0, 0, 20, 300, 1, 7], dtype=torch.int32, device=DEV),
              top_p=torch.tensor([1.0, 0.9, 1.0, 0.8, 1.0, 0.95], device=DEV),
              min_p=torch.tensor([0.0, 0.0, 0.05, 0.0, 0.0, 0.2], device=DEV))
    _check_verify(n, B, 6000, *_verify_case(n, B, 6000, 8, **kw), kw)


def test_verify_same_distributions_accepts_everything():
    """p = q: every draft is accepted, whatever the uniform below 1."""
    n, B, V = 3, 9, 5000
    z, t, tok, cut, u = _verify_case(n, B, V, 5, near=0.0, kind="flat", top_p=0.9)
    u[:, :B - 1] = 1 - 2.0 ** -24
    acc = _check_verify(n, B, V, z, t, tok, cut, u, dict(top_p=0.9))
    assert acc == [B - 1] * n


def test_verify_disjoint_masked_and_out_of_range():
    """Target rows that give the draft no mass, rows masked throughout on either side, drafts that
    are no tokens."""
    n, B, V = 5, 4, 3000
    z, t, tok, cut, u = _verify_case(n, B, V, 77)
    t[0, 0] = -np.inf
    t[0, 0, 1234] = 0.5                 # a target of one token
    t[1, 1] = -np.inf                   # a target row masked throughout
    z[2 * B + 1] = -np.inf              # a draft row masked throughout
    tok, cut = hdf.sample_truncated(z, _u(n * B, 6), rows_per_seq=B)
    assert int(tok[2 * B + 1]) == -1
    tok[3 * B + 2] = V
    tok[4 * B + 1] = -7
    u[1, 0] = 0.0
    acc = _check_verify(n, B, V, z, t, tok, cut, u, {})
    assert acc[2] == 0 and acc[3] <= 1 and acc[4] == 0


def test_verify_many_sequences():
    """More sequences than a workgroup has threads: the commit offsets run on."""
    n, B, V = 700, 3, 64
    kw = dict(top_k=20)
    _check_verify(n, B, V, *_verify_case(n, B, V, 13, kind="flat", **kw), kw)


# ------------------------------------------------------------- streams, graphs, repetition

def test_another_stream_and_given_workspace():
    z = _logits(3, 7000, 5)
    u = _u(3, 5)
    want = hdf.sample_truncated(z, u, top_p=0.9)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ws = torch.empty(max(1, hdf.lib().hdf_sample_truncated_workspace(3, 7000, 0)),
                     dtype=torch.uint8, device=DEV)
    s.wait_stream(torch.cuda.current_stream())
    got = hdf.sample_truncated(z, u, top_p=0.9, ws=ws, stream=s)
    top = hdf.top_logits(z, 9, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got[0], want[0]) and all(torch.equal(a, b) for a, b in zip(got[1], want[1]))
    assert all(torch.equal(a, b) for a, b in zip(top, hdf.top_logits(z, 9)))


def test_two_streams_at_once():
    a, b = _logits(64, 30000, 1), _logits(64, 30000, 2, kind="flat")
    u = _u(64, 3)
    want = [hdf.sample_truncated(x, u, top_p=0.9) for x in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = [hdf.sample_truncated(x, u, top_p=0.9, stream=s) for x, s in zip((a, b), streams)]
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g[0], w[0]) and torch.equal(g[1].lse, w[1].lse)


def test_captured_tail_replays():
    """Draw, verify and record in one graph, replayed over changing inputs with eager work and
    synchronizations between: every replay equals the eager calls."""
    n, B, V = 4, 6, 9001
    kw = dict(top_k=60, top_p=0.95)
    z = torch.empty(n * B, V, device=DEV)
    t = torch.empty(n, B, V, device=DEV)
    u0, u1 = torch.empty(n * B, device=DEV), torch.empty(n, B, device=DEV)

    def fill(seed):
        c = _verify_case(n, B, V, seed, **kw)
        z.copy_(c[0]), t.copy_(c[1]), u1.copy_(c[4]), u0.copy_(_u(n * B, seed))

    def step():
        tok, cut = hdf.sample_truncated(z, u0, rows_per_seq=B, **kw)
        res = hdf.accept_truncated(tok[1:], z[1:], tuple(x[1:] for x in cut), t, u1, K=B - 1,
                                   draft_stride=B, out=out, **kw)
        return (tok, *cut, *res, *hdf.top_logits(t.view(n * B, V), 16))

    out = tuple(torch.zeros(m, dtype=torch.int32, device=DEV) for m in (n, n, n + 1, n * B))
    fill(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = step()
    for seed in (1, 50, 51, 52):
        fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in res]
        for o in out:
            o.zero_()
        want = step()
        torch.cuda.synchronize()
        live = int(want[7][-1])
        for i, (g, w) in enumerate(zip(got, want)):
            if i == 8:
                g, w = g[:live], w[:live]
            assert torch.equal(g, w), (seed, i)


def test_same_call_same_bits():
    z = _logits(40, 60000, 6, kind="flat")
    u = _u(40, 6)
    first = hdf.sample_truncated(z, u, temperature=1.2, top_p=0.97)
    for _ in range(5):
        again = hdf.sample_truncated(z, u, temperature=1.2, top_p=0.97)
        assert torch.equal(first[0], again[0])
        assert all(torch.equal(a, b) for a, b in zip(first[1], again[1]))
