"""Distillation from top logits on the GPU, forward and backward, against the float64 oracle.

Tolerances.  The kernels' exponentials are 32-bit: an exponent a (base 2) is off by 2^-23 |a| at
the most (a product and a difference rounded), which weighs a term of 2^a by |a| 2^a <= 0.54, and
the instruction by an ulp, 2^-23; a thread adds 32 of them in fp32, 31 * 2^-24 at the worst, and
the rest is 64-bit.  A sum is thus right to REL = (0.54 * 0.7 + 1 + 15.5) * 2^-23 < 2.1e-6, its
logarithm to the same absolutely.  kl holds two such logarithms at most (q and q_rest):
2 REL (1 + p_rest) + half an ulp; ce one and half an ulp.  A gradient's positive parts (q, its
tail factor p_rest / q_rest, p) are each right to 3 REL + 4 * 2^-23 relative, and the result is
rounded once to the logits' type."""
import numpy as np
import pytest
import torch

from oracle import distill as od
from paper_2606_26744_amd import hdf
from paper_2606_26744_amd.distill import distill_loss

pytestmark = pytest.mark.gpu
DEV = "cuda"
REL = 2.1e-6
GREL = 3 * REL + 4 * 2.0 ** -23


def _np(t):
    return None if t is None else t.detach().cpu().double().numpy()


def _case(n, B, P, K, V, seed, dtype=torch.float32, rest=True, labels=True, T=1.0, ld=None, offset=0):
    g = torch.Generator().manual_seed(seed)
    ld = ld or V
    buf = torch.full((n * B * ld + offset + 8,), 55.0, dtype=dtype, device=DEV)
    z = torch.as_strided(buf, (n * B, V), (ld, 1), offset)
    zc = torch.randn(n * B, V, generator=g) * 2
    zc[:, torch.randint(0, V, (min(V, 9),), generator=g)] += 6
    z.copy_(zc)
    t = zc.view(n, B, V)[:, 1:P + 1].reshape(n * P, V) + torch.randn(n * P, V, generator=g) * 0.7
    ids, val, r = hdf.top_logits(t.to(DEV), K, temperature=T)
    lab = torch.randint(0, V, (n, B - 1), generator=g, dtype=torch.int32).to(DEV) if labels else None
    return dict(z=z, ids=ids.view(n, P, K), val=val.view(n, P, K),
                rest=r.view(n, P) if rest else None, lab=lab)


def _parts(c, B, T, wk, wc):
    """Sum of the gradient's parts by magnitude: what its relative errors refer to."""
    z = _np(c["z"])
    ids, val, rest = c["ids"].tolist(), _np(c["val"]), _np(c["rest"])
    n, P = len(ids), len(ids[0])
    mag = np.zeros_like(z)
    V = z.shape[1]
    for s in range(n):
        for k in range(1, B):
            x = z[s * B + k]
            if x.max() == -np.inf:
                continue
            if k <= P:
                toks, p, pr = od.teacher(ids[s][k - 1], val[s][k - 1],
                                         None if rest is None else rest[s][k - 1], V, T)
                if p is not None:
                    q = od._softmax(x / T)
                    out = q.sum() - q[toks].sum() if len(toks) else 1.0
                    m = q * (1 + (pr / out if pr > 0 else 0))
                    m[toks] = q[toks] + p
                    mag[s * B + k] += abs(wk[s][k - 1]) / T * m
            if c["lab"] is not None and 0 <= int(c["lab"][s, k - 1]) < V:
                m = od._softmax(x)
                m[int(c["lab"][s, k - 1])] += 1
                mag[s * B + k] += abs(wc[s][k - 1]) * m
    return mag


def _check(c, B, T=1.0, alpha=0.5, g_loss=(0.0, 0.0, 1.0), g_kl=None, g_ce=None, d_logits=None):
    n, P, K = c["ids"].shape
    kl, ce, loss, saved = hdf.distill_forward(c["z"], c["ids"], c["val"], c["rest"], c["lab"], B=B,
                                              temperature=T, alpha=alpha)
    up = [None if x is None else torch.as_tensor(x, dtype=torch.float32, device=DEV)
          for x in (g_loss, g_kl, g_ce)]
    d = hdf.distill_backward(c["z"], c["ids"], c["lab"], saved, B=B, temperature=T, alpha=alpha,
                             grad_loss=up[0], grad_kl=up[1], grad_ce=up[2], d_logits=d_logits)
    torch.cuda.synchronize()
    gl = (0, 0, 0) if g_loss is None else [float(np.float32(x)) for x in g_loss]
    wkl, wce, wloss, wgrad = od.distill(_np(c["z"]), c["ids"].tolist(), _np(c["val"]),
                                        _np(c["rest"]), None if c["lab"] is None else c["lab"].cpu(),
                                        B, T, alpha, gl, _np(up[1]), _np(up[2]))
    half = 2.0 ** -24
    err = np.abs(_np(kl) - wkl)
    assert (err <= 4 * REL + half * np.abs(wkl)).all(), err.max()
    if ce is not None:
        err = np.abs(_np(ce) - wce)
        assert (err <= REL + half * np.abs(wce)).all(), err.max()
    bound = T * T * 4 * REL * (1 + alpha) + REL + 2 * half * np.abs(wloss)
    assert (np.abs(_np(loss) - wloss) <= bound).all(), (loss, wloss)
    Pn = P * n
    wk = (gl[0] + alpha * gl[2]) * T * T / Pn + (np.zeros((n, P)) if g_kl is None else _np(up[1]))
    has = max(1, 0 if c["lab"] is None else int(((c["lab"] >= 0) & (c["lab"] < c["z"].shape[1])).sum()))
    wc = (gl[1] + gl[2]) / has + (np.zeros((n, B - 1)) if g_ce is None else _np(up[2]))
    mag = _parts(c, B, float(np.float32(T)), wk, wc)
    step = torch.finfo(c["z"].dtype).eps / 2
    err = np.abs(_np(d) - wgrad)
    tol = (GREL * mag) * (1 + step) + step * np.abs(wgrad) + 1e-37
    assert (err <= tol).all(), (np.argwhere(err > tol)[:4], err.max())
    return kl, ce, loss, d


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rest,labels,T", [(True, True, 1.0), (True, False, 2.0), (False, True, 2.0),
                                           (False, False, 1.0), (True, True, 0.5)])
def test_losses_and_gradients(dtype, rest, labels, T):
    c = _case(3, 6, 3, 20, 9001, 5, dtype, rest, labels, T)
    _check(c, 6, T)


@pytest.mark.parametrize("n,B,P,K,V", [(1, 2, 1, 1, 1), (1, 2, 1, 4, 2), (2, 3, 2, 3, 5),
                                       (1, 3, 1, 64, 64), (2, 5, 4, 7, 8191), (1, 4, 3, 128, 8193),
                                       (1, 3, 2, 1024, 16411), (40, 2, 1, 5, 300), (1, 40, 39, 9, 77),
                                       (1, 2, 1, 50, 151937)])
def test_sizes(n, B, P, K, V):
    for dtype in (torch.float32, torch.bfloat16):
        _check(_case(n, B, P, K, V, V + K, dtype, ld=V + 3, offset=1), B)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", range(8))
def test_every_alignment_of_logits_and_gradients(offset, dtype):
    """Logits and gradients that start at different elements of a vector, and the columns between
    the gradients' rows left as they were."""
    n, B, V = 2, 3, 4099
    c = _case(n, B, 2, 9, V, offset, dtype, ld=V + 2, offset=offset)
    for shift in (offset, 0, 3):
        ldd = V + 5
        buf = torch.full((n * B * ldd + shift + 8,), 9.0, dtype=dtype, device=DEV)
        d = torch.as_strided(buf, (n * B, V), (ldd, 1), shift)
        _check(c, B, d_logits=d)
        mask = torch.ones_like(buf, dtype=torch.bool)
        torch.as_strided(mask, (n * B, V), (ldd, 1), shift).fill_(False)
        assert (buf[mask] == 9.0).all()


def test_rows_more_than_32_bits_apart():
    """Logits and gradients whose offsets in elements pass 2^32."""
    n, B, V, ld = 1, 3, 4003, 2 ** 31 + 8
    c = _case(n, B, 2, 9, V, 3, torch.bfloat16)
    z, d = (torch.as_strided(torch.empty(2 * ld + V, dtype=torch.bfloat16, device=DEV), (B, V), (ld, 1))
            for _ in range(2))
    z.copy_(c["z"])
    c["z"] = z
    _check(c, B, d_logits=d)


def test_every_upstream_gradient():
    n, B, P = 3, 5, 2
    c = _case(n, B, P, 10, 5000, 2)
    g = np.random.default_rng(1)
    gk, gc = g.normal(size=(n, P)), g.normal(size=(n, B - 1))
    _check(c, B, g_loss=(1.0, 0.0, 0.0))
    _check(c, B, g_loss=(0.0, 1.0, 0.0))
    _check(c, B, g_loss=(0.3, -0.2, 2.0), g_kl=gk, g_ce=gc)
    _check(c, B, g_loss=None, g_kl=gk)
    _check(c, B, g_loss=None, g_ce=gc)
    _, _, _, d = _check(c, B, g_loss=None)
    assert not d.any()


def test_lists_with_gaps_repeats_and_labels_among_them():
    """Ids outside the vocabulary and repeated ones, teacher logits of -inf, an empty list, labels
    that are listed, unlisted and to be ignored."""
    n, B, P, K, V = 2, 5, 4, 40, 3001
    c = _case(n, B, P, K, V, 7)
    ids, val, lab = c["ids"], c["val"], c["lab"]
    ids[0, 0, 5:9] = ids[0, 0, 2]
    ids[0, 1, 7] = -1
    ids[0, 1, 8] = V
    ids[0, 1, 9] = 2 ** 31 - 1
    ids[1, 0] = -1
    val[0, 2, 3:] = -np.inf
    ids[1, 2] = ids[1, 2, 0]
    lab[0, 0] = ids[0, 0, 2]
    lab[0, 1] = ids[0, 1, 0]
    lab[0, 2] = -100
    lab[1, 3] = V
    _check(c, B)
    c["rest"] = None
    val[1, 1] = -np.inf
    _check(c, B, T=2.0)
    lab.fill_(-100)
    _, ce, loss, _ = _check(c, B)
    assert not ce.any() and float(loss[1]) == 0


def test_masked_students():
    """Masked student logits outside and inside the list, the type's lowest value as a mask."""
    n, B, P, K, V = 1, 5, 4, 12, 2500
    c = _case(n, B, P, K, V, 9)
    z = c["z"]
    keep = torch.zeros(V, dtype=torch.bool, device=DEV)
    keep[c["ids"][0, 0].long()] = True
    keep[::7] = True
    z[1, ~keep] = -np.inf
    z[2, 1000:] = torch.finfo(torch.float32).min
    c["val"][0, 1, 0] = -np.inf
    z[3, ::2] = -np.inf
    c["lab"][0, 0] = c["ids"][0, 0, 0]
    c["lab"][0, 1] = 3
    c["lab"][0, 2] = 1
    # Row 2's list holds tokens of the lowest value: their log-probabilities are beyond any sum.
    inside = c["ids"][0, 1] < 1000
    c["ids"][0, 1][~inside] = -1
    c["ids"][0, 2][c["ids"][0, 2] % 2 == 0] = -1
    c["rest"][0, 1] = -2.0
    _check(c, B)


@pytest.mark.parametrize("T", [1.0, 0.5])
def test_students_far_from_zero(T):
    """Rows of the type's lowest value throughout, and rows whose greatest logit is so large that its
    product with log2(e) / T rounds to no small part of an octave: differences of logits are what
    counts."""
    n, B, P, K, V = 1, 6, 5, 12, 3001
    c = _case(n, B, P, K, V, 14, T=T)
    z = c["z"]
    z[1] = torch.finfo(torch.float32).min
    z[2] += 2.0 ** 19
    z[3] = (z[3] - 4) * 2.0 ** 20 * T
    z[4] -= 2.0 ** 17
    z[5] = 1e30
    c["ids"][0, 2] = z[3].topk(K).indices.int()   # the others are beyond any sum
    c["rest"][0, 2] = -np.inf
    _check(c, B, T)


@pytest.mark.parametrize("T", [1.0, 0.125])
def test_unlisted_columns_far_below_the_listed_ones(T):
    """A student all of whose unlisted columns vanish beside the listed ones: the bucket's divergence
    is finite, and its gradient is spread over them by their own softmax, by formula in 64 bits."""
    n, B, P, K, V = 2, 4, 3, 6, 700
    for dtype in (torch.float32, torch.bfloat16):
        c = _case(n, B, P, K, V, 21, dtype, labels=False, T=T)
        z = c["z"].view(n, B, V)
        for s in range(n):
            for k in range(1, P + 1):
                z[s, k, c["ids"][s, k - 1].long()] += 200.0 * (s + 1)
        c["rest"][:] = c["val"][:, :, 0] / T - 1.0       # a bucket of weight
        kl, _, _, saved = hdf.distill_forward(c["z"], c["ids"], c["val"], c["rest"], B=B, temperature=T)
        d = hdf.distill_backward(c["z"], c["ids"], None, saved, B=B, temperature=T,
                                 grad_kl=torch.ones(n, P, device=DEV))
        step = torch.finfo(dtype).eps / 2
        for s in range(n):
            for k in range(1, P + 1):
                x = _np(z[s, k]) / T
                toks, p, pr = od.teacher(c["ids"][s, k - 1].tolist(), _np(c["val"])[s, k - 1],
                                         float(c["rest"][s, k - 1]), V, T)
                want, grad = od.slot_kl(_np(z[s, k]), c["ids"][s, k - 1].tolist(),
                                        _np(c["val"])[s, k - 1], float(c["rest"][s, k - 1]), T)
                assert np.isfinite(want)
                assert abs(float(kl[s, k - 1]) - want) <= 4 * REL + 2.0 ** -24 * abs(want)
                inside = np.zeros(V, bool)
                inside[toks] = True
                far = np.where(inside, -np.inf, x)
                spread = np.exp(far - far.max())
                spread /= spread.sum()
                grad = -pr * spread / T              # q itself is beyond 64 bits, or next to it
                q = np.exp(x - x.max())
                grad[inside] = ((q / q.sum())[inside] - p[np.argsort(toks)]) / T
                got = _np(d.view(n, B, V)[s, k])
                mag = np.where(inside, 2.0, pr * spread) / T
                assert (np.abs(got - grad) <= GREL * mag * (1 + step) + step * np.abs(grad) + 1e-37).all()


@pytest.mark.parametrize("n", [32, 33, 70])
def test_means_over_few_and_many_slots(n):
    """Slots that one launch counts and more, over a workspace of arbitrary contents, used again."""
    B, P, K, V = 9, 8, 70, 301
    c = _case(n, B, P, K, V, n)
    _check(c, B)
    ws = torch.full((hdf.lib().hdf_distill_workspace(n, B, V, 0),), 255, dtype=torch.uint8, device=DEV)
    args = (c["z"], c["ids"], c["val"], c["rest"], c["lab"])
    want = hdf.distill_forward(*args, B=B)
    for _ in range(3):
        got = hdf.distill_forward(*args, B=B, ws=ws)
        assert all(torch.equal(g, w) for g, w in zip(got[:3], want[:3]))


@pytest.mark.parametrize("K", [63, 64, 65, 255, 256, 257, 700])
def test_list_lengths(K):
    _check(_case(2, 3, 2, K, 2003, K), 3)


def test_student_that_gives_a_listed_token_no_mass():
    c = _case(1, 3, 2, 5, 400, 3)
    c["z"][1, c["ids"][0, 0, 2].long()] = -np.inf
    c["z"][2] = -np.inf
    kl, ce, loss, saved = hdf.distill_forward(c["z"], c["ids"], c["val"], c["rest"], c["lab"], B=3)
    assert torch.isposinf(kl).all() and torch.isposinf(loss[0]) and torch.isposinf(ce[0, 1])
    d = hdf.distill_backward(c["z"], c["ids"], c["lab"], saved, B=3,
                             grad_kl=torch.ones(1, 2, device=DEV))
    assert torch.isfinite(d).all()
    p = od.teacher(c["ids"][0, 1].tolist(), _np(c["val"])[0, 1], float(c["rest"][0, 1]), 400, 1.0)
    want = np.zeros(400)
    want[p[0]] = -p[1]
    np.testing.assert_allclose(_np(d)[2], want, atol=1e-6)


def test_nan_reaches_the_losses_and_gradients_of_its_slot_alone():
    c = _case(2, 4, 3, 6, 700, 4)
    c["z"][1, 333] = float("nan")
    c["val"][1, 1, 2] = float("nan")
    c["rest"][1, 2] = float("nan")
    kl, ce, loss, saved = hdf.distill_forward(c["z"], c["ids"], c["val"], c["rest"], c["lab"], B=4)
    assert torch.isnan(kl).tolist() == [[True, False, False], [False, True, True]]
    assert torch.isnan(ce).tolist() == [[True, False, False], [False, False, False]]
    assert torch.isnan(loss).all()
    d = hdf.distill_backward(c["z"], c["ids"], c["lab"], saved, B=4,
                             grad_loss=torch.ones(3, device=DEV))
    assert torch.isnan(d).any(1).tolist() == [False, True, False, False, False, False, True, True]


def test_rows_past_the_supervised_slots_are_zero():
    c = _case(2, 6, 2, 6, 1001, 8, labels=False)
    d = torch.full((12, 1001), 7.0, device=DEV)
    _check(c, 6, d_logits=d)
    assert not d.view(2, 6, 1001)[:, [0, 3, 4, 5]].any()


def test_empty_batch():
    z = torch.empty(0, 50, device=DEV)
    ids, val = torch.empty(0, 2, 4, dtype=torch.int32, device=DEV), torch.empty(0, 2, 4, device=DEV)
    kl, ce, loss, saved = hdf.distill_forward(z, ids, val, B=3)
    assert kl.shape == (0, 2) and not loss.any()
    assert hdf.distill_backward(z, ids, None, saved, B=3).shape == (0, 50)


def test_autograd_matches_the_direct_call_and_differences():
    n, B, P, T, alpha = 2, 5, 3, 2.0, 0.7
    c = _case(n, B, P, 16, 3000, 12, T=T)
    z = c["z"].clone().requires_grad_()
    args = (c["ids"], c["val"], c["rest"], c["lab"])
    loss, kl, ce = distill_loss(z, *args, B=B, temperature=T, alpha=alpha)
    (loss[2] * 1.5 + kl.sum() * 0.25 - (ce[0] * 0.1).sum()).backward()
    kl_, ce_, loss_, saved = hdf.distill_forward(c["z"], *args, B=B, temperature=T, alpha=alpha)
    gc = torch.zeros(n, B - 1, device=DEV)
    gc[0] = -0.1
    want = hdf.distill_backward(c["z"], c["ids"], c["lab"], saved, B=B, temperature=T, alpha=alpha,
                                grad_loss=torch.tensor([0.0, 0.0, 1.5], device=DEV),
                                grad_kl=torch.full((n, P), 0.25, device=DEV), grad_ce=gc)
    assert torch.equal(loss, loss_) and torch.equal(kl, kl_) and torch.equal(ce, ce_)
    assert torch.equal(z.grad, want)
    # Central differences of the summed kl along a direction u of unit entries: the loss is right to
    # n P (4 REL + half an ulp of kl) and the third derivative along u is at most 8 n P / T^3.
    u = torch.sign(torch.randn(z.shape, generator=torch.Generator().manual_seed(2))).to(DEV)
    h = 2.0 ** -4
    f = [float(hdf.distill_forward(c["z"] + s * h * u, *args, B=B, temperature=T)[0].double().sum())
         for s in (1, -1)]
    _, _, _, saved = hdf.distill_forward(c["z"], *args, B=B, temperature=T)
    g = hdf.distill_backward(c["z"], c["ids"], c["lab"], saved, B=B, temperature=T,
                             grad_kl=torch.ones(n, P, device=DEV))
    slope = float((g.double() * u.double()).sum())
    tol = n * P * ((4 * REL + 2.0 ** -24 * 10 + 2.0 ** -24 * 20) / h + 8 / T ** 3 * h * h / 6 + 2 * GREL)
    assert abs((f[0] - f[1]) / (2 * h) - slope) <= tol


def test_autograd_leaves_the_rest_alone():
    """No gradient asked for, parts of the outputs unused, a second use of the same leaf, 16-bit
    logits behind a product."""
    c = _case(2, 4, 2, 8, 600, 3)
    args = (c["ids"], c["val"], c["rest"], c["lab"])
    with torch.no_grad():
        loss, _, _ = distill_loss(c["z"], *args, B=4)
    assert not loss.requires_grad
    w = torch.randn(32, 600, device=DEV, generator=torch.Generator(DEV).manual_seed(1)) * 0.3
    w.requires_grad_()
    x = torch.randn(8, 32, device=DEV, generator=torch.Generator(DEV).manual_seed(2))
    zb = (x @ w).bfloat16()
    loss, kl, ce = distill_loss(zb, *args, B=4)
    g, = torch.autograd.grad(loss[2] + kl[0, 0], w)
    assert g.shape == w.shape and torch.isfinite(g).all() and g.any()
    _, _, _, saved = hdf.distill_forward(zb.detach(), *args, B=4)
    gk = torch.zeros(2, 2, device=DEV)
    gk[0, 0] = 1
    d = hdf.distill_backward(zb.detach(), c["ids"], c["lab"], saved, B=4, grad_kl=gk,
                             grad_loss=torch.tensor([0.0, 0.0, 1.0], device=DEV))
    # One product of 8 terms on both sides, the same operands.
    torch.testing.assert_close(g, x.t() @ d.float(), rtol=1e-5, atol=1e-6)


def test_record_and_train_together():
    """The teacher's side and the student's in a row, as a training program runs them: descending
    the gradient of blocks that stand at the teacher does nothing, and elsewhere the gradient's
    rows sum to zero."""
    n, B, P, K, V, T = 2, 4, 3, 32, 4097, 2.0
    g = torch.Generator().manual_seed(6)
    t = (torch.randn(n * B, V, generator=g) * 2).to(DEV)
    ids, val, rest = hdf.top_logits(t, K, temperature=T)
    sel = torch.arange(n * B).view(n, B)[:, 1:P + 1].reshape(-1).to(DEV)
    lists = [x[sel].view(n, P, *x.shape[1:]).contiguous() for x in (ids, val, rest)]
    z = t.clone().requires_grad_()
    loss, kl, _ = distill_loss(z, *lists, B=B, temperature=T)
    loss[0].backward()
    assert kl.abs().max() <= 8 * REL
    assert z.grad.abs().max() <= 2 * GREL
    y = (t + torch.randn(n * B, V, generator=g).to(DEV)).requires_grad_()
    loss, kl, _ = distill_loss(y, *lists, B=B, temperature=T)
    kl.sum().backward()
    # A divergence of two distributions is positive (Gibbs); nothing says by how much here, and the
    # kernel knows it to 4 REL.
    assert (kl > 4 * REL).all()
    assert y.grad.double().sum(1).abs().max() <= 4 * GREL


def test_captured_step_replays():
    n, B, P, K, V = 3, 4, 3, 8, 5001
    c = _case(n, B, P, K, V, 1)
    z = c["z"]
    g = torch.tensor([0.0, 0.0, 1.0], device=DEV)

    def step():
        kl, ce, loss, saved = hdf.distill_forward(z, c["ids"], c["val"], c["rest"], c["lab"], B=B)
        return kl, ce, loss, hdf.distill_backward(z, c["ids"], c["lab"], saved, B=B, grad_loss=g)

    # An eager graph over the same logits is alive while the step is captured.
    leaf = z.clone().requires_grad_()
    alive = distill_loss(leaf, c["ids"], c["val"], c["rest"], c["lab"], B=B)[0][2]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = step()
    for seed in range(4):
        z.copy_(torch.randn(n * B, V, generator=torch.Generator().manual_seed(seed)) * 2)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in res]
        for a, b in zip(got, step()):
            assert torch.equal(a, b), seed
    alive.backward()
    assert torch.isfinite(leaf.grad).all()


def test_another_stream_and_repetition():
    c = _case(4, 8, 7, 32, 32003, 2)
    args = (c["z"], c["ids"], c["val"], c["rest"], c["lab"])
    want = hdf.distill_forward(*args, B=8)
    dwant = hdf.distill_backward(c["z"], c["ids"], c["lab"], want[3], B=8,
                                 grad_loss=torch.ones(3, device=DEV))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    up = torch.ones(3, device=DEV)
    torch.cuda.synchronize()
    for _ in range(3):
        got = hdf.distill_forward(*args, B=8, stream=s)
        d = hdf.distill_backward(c["z"], c["ids"], c["lab"], got[3], B=8, grad_loss=up, stream=s)
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got[:3], want[:3]))
        assert torch.equal(d, dwant)
