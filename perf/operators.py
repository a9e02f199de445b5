"""Rows of logits cut to the head of their distribution, as cases that can be timed and checked:
truncated draws (temperature, top-k, top-p, min-p), the speculative verification of such draws,
the extraction of a row's top logits, and the distillation from a teacher's stored top logits,
forward and backward.

Where `own` is false, run() computes a case with elementary torch operations; where it is true
it makes the library's calls.  listed() gives the sizes that stand for the operators, draw()
more of the same ranges; prepare() makes what a program holds before the call, exact() the same
outputs in 64 bits from the definitions (cuts by bisection, gradients by differentiation).

The order of a row's entries is by value, largest first, ties to the lowest index; an entry of
-inf is masked.  All distributions are cut to a first part of that order.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
F64 = torch.float64
NINF = float("-inf")


# ------------------------------------------------------------------------------ cases

def listed():
    V = 129280
    return [
        # One sequence's next token while the others wait: a launch's latency.
        dict(name="draw_one", kind="draw", rows=1, per=1, V=V, dtype="f32", shape="peaked",
             settings="mixed", mask=0.0, ld_extra=0),
        # Every slot of a round's blocks drawn, eight sequences with settings of their own.
        dict(name="draw_round", kind="draw", rows=128, per=16, V=V, dtype="f32", shape="peaked",
             settings="mixed", mask=0.0, ld_extra=0),
        # A warm (high temperature) nucleus over flat logits: much of the vocabulary is kept.
        dict(name="draw_flat", kind="draw", rows=60, per=15, V=32003, dtype="f32", shape="flat",
             settings="warm", mask=0.0, ld_extra=0),
        # A full serving batch of 64 blocks under a plain nucleus, logits kept in 16 bits.
        dict(name="draw_batch", kind="draw", rows=1024, per=16, V=V, dtype="bf16", shape="peaked",
             settings="nucleus", mask=0.0, ld_extra=0),
        # Verification of a round of eight sequences.
        dict(name="verify_round", kind="verify", n_seq=8, B=16, V=V, dtype="f32", shape="peaked",
             settings="mixed"),
        # A short block of one sequence, the target's logits in 16 bits.
        dict(name="verify_one", kind="verify", n_seq=1, B=8, V=32000, dtype="bf16", shape="peaked",
             settings="nucleus"),
        # A teacher's top logits recorded for the blocks of one small step.
        dict(name="top_small", kind="top", rows=37, V=32003, dtype="f32", K=20, temperature=1.0,
             ld_extra=5),
        # The same for a batch of long blocks, from 16-bit logits.
        dict(name="top_batch", kind="top", rows=960, V=V, dtype="bf16", K=128, temperature=2.0,
             ld_extra=0),
        # The objective alone (an evaluation pass) over a few blocks.
        dict(name="distill_eval", kind="distill", n_seq=8, B=16, P=15, V=V, dtype="f32", K=64,
             temperature=1.0, rest=True, labels=True, backward=False),
        # ... of 16-bit logits at a softer temperature, the teacher renormalised over its list.
        dict(name="distill_eval_soft", kind="distill", n_seq=4, B=16, P=2, V=32003, dtype="bf16",
             K=20, temperature=2.0, rest=False, labels=True, backward=False),
        # A small training step: the objective and the gradient of every logit.
        dict(name="distill_step", kind="distill", n_seq=4, B=8, P=7, V=32000, dtype="f32", K=32,
             temperature=1.0, rest=True, labels=True, backward=True),
        # A training step over a full batch of blocks.
        dict(name="distill_step_batch", kind="distill", n_seq=64, B=16, P=15, V=V, dtype="bf16",
             K=64, temperature=1.0, rest=True, labels=True, backward=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["draw", "draw", "verify", "top", "distill", "distill"])
    V = _log_int(rng, 4001, 151936)
    dtype = rng.choice(["f32", "f32", "bf16"])
    most = 1024 * 129280 // V
    if kind == "draw":
        per = rng.choice([1, 4, 7, 8, 15, 16])
        rows = per * _log_int(rng, 1, max(1, min(1024, most // 2) // per))
        return dict(kind=kind, rows=rows, per=per, V=V, dtype=dtype,
                    shape=rng.choice(["peaked", "peaked", "flat"]),
                    settings=rng.choice(["mixed", "mixed", "nucleus", "top_k", "warm", "open"]),
                    mask=rng.choice([0.0, 0.0, 0.3, 0.9]), ld_extra=rng.choice([0, 0, 3, 64]))
    if kind == "verify":
        B = rng.choice([2, 4, 7, 8, 16, 16])
        return dict(kind=kind, n_seq=_log_int(rng, 1, max(1, min(32, most // (2 * B)))), B=B, V=V,
                    dtype=dtype, shape=rng.choice(["peaked", "peaked", "flat"]),
                    settings=rng.choice(["mixed", "nucleus", "top_k", "open"]))
    if kind == "top":
        return dict(kind=kind, rows=_log_int(rng, 1, min(960, most // 2)), V=V, dtype=dtype,
                    K=_log_int(rng, 1, 256), temperature=rng.choice([1.0, 1.0, 2.0, 4.0]),
                    ld_extra=rng.choice([0, 0, 5, 32]))
    B = rng.choice([2, 5, 8, 16, 16])
    return dict(kind=kind, n_seq=_log_int(rng, 1, max(1, min(48, most // (2 * B)))), B=B,
                P=rng.randint(1, B - 1), V=V, dtype=dtype, K=_log_int(rng, 1, 256),
                temperature=rng.choice([1.0, 1.0, 2.0]), rest=rng.random() < 0.6,
                labels=rng.random() < 0.8, backward=rng.random() < 0.6)


# ----------------------------------------------------------------------------- inputs

class _Draws:
    """Seeded draws on the GPU, one generator per tensor name."""

    def __init__(self, seed):
        self.seed = int(seed)

    def _gen(self, name):
        g = torch.Generator(device=DEV)
        k = 0
        for ch in name:
            k = (k * 131 + ord(ch)) % 1_000_003
        g.manual_seed((self.seed * 1_000_003 + k) & ((1 << 62) - 1))
        return g

    def normal(self, name, shape, std=1.0):
        return torch.randn(*shape, generator=self._gen(name), device=DEV).mul_(std)

    def uniform(self, name, shape):
        return torch.rand(*shape, generator=self._gen(name), device=DEV)

    def ints(self, name, shape, hi):
        return torch.randint(0, hi, tuple(shape), generator=self._gen(name), device=DEV)


def _logits(g, name, rows, V, shape, ld_extra=0):
    """Logits of `rows` positions: noise of an LM head's scale and, for peaked rows, a few dozen
    plausible tokens that stand out of it."""
    ld = V + ld_extra
    if shape == "flat":
        return g.normal(name, (rows, ld), 1.3)
    z = g.normal(name, (rows, ld), 1.8)
    head = g.ints(name + ".head", (rows, 48), V)
    return z.scatter_reduce_(1, head, g.uniform(name + ".lift", (rows, 48)).mul_(9.0).add_(5.0),
                             "amax")


def _cast(z, dtype):
    return z.to(torch.bfloat16) if dtype == "bf16" else z


def _settings(g, kind, n):
    """Sampling settings as a serving batch holds them: one value for all sequences, or a
    tensor with one a sequence."""
    def pick(name, values, dtype):
        t = torch.tensor(values, dtype=dtype, device=DEV)
        return t[g.ints(name, (n,), len(values))].contiguous()

    if kind == "mixed":
        return dict(temperature=pick("temperature", [0.6, 0.7, 0.8, 1.0, 1.0, 0.0], torch.float32),
                    top_k=pick("top_k", [0, 20, 50, 100, 0], torch.int32),
                    top_p=pick("top_p", [1.0, 0.8, 0.9, 0.95], torch.float32),
                    min_p=pick("min_p", [0.0, 0.0, 0.02, 0.1], torch.float32))
    one = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
    if kind == "nucleus":
        one["top_p"] = 0.95
    elif kind == "top_k":
        one.update(temperature=0.8, top_k=50)
    elif kind == "warm":
        one.update(temperature=1.5, top_p=0.95)
    return one


def _row_settings(s, rows, per):
    """The four settings as a column each, one entry a row, in the order temperature, top_k,
    top_p, min_p (32-bit values widened to 64 bits)."""
    out = []
    for key in ("temperature", "top_k", "top_p", "min_p"):
        v = s[key]
        if not torch.is_tensor(v):
            v = torch.full((rows,), v, dtype=torch.float32, device=DEV)
        else:
            v = v.repeat_interleave(per)[:rows]
        out.append(v.to(F64).unsqueeze(1))
    return out


def prepare(case, seed):
    c, g, kind = case, _Draws(seed), case["kind"]
    s = dict(case=c)
    if kind == "draw":
        z = _logits(g, "logits", c["rows"], c["V"], c["shape"], c["ld_extra"])
        if c["mask"]:
            z.masked_fill_(g.uniform("mask", z.shape) < c["mask"], NINF)
        s["logits"] = _cast(z, c["dtype"])[:, :c["V"]]
        s["settings"] = _settings(g, c["settings"], -(-c["rows"] // c["per"]))
        s["uniforms"] = g.uniform("u", (c["rows"],))
    elif kind == "verify":
        n, B, V = c["n_seq"], c["B"], c["V"]
        s["settings"] = _settings(g, c["settings"], n)
        # The drafter's rows of a block (slot 0 holds the anchor); the target's stand near them.
        z = _logits(g, "draft", n * B, V, c["shape"])
        t = g.normal("target", (n, B, V), 0.6)
        t[:, :B - 1] += z.view(n, B, V)[:, 1:]
        t[:, B - 1] += z.view(n, B, V)[:, 0]
        s["draft_logits"], s["target_logits"] = z, _cast(t, c["dtype"])
        cut = _cut(z, _row_settings(s["settings"], n * B, B))
        s["draft_cut"] = (cut["kept"], cut["cut_logit"], cut["cut_index"], cut["lse"])
        s["draft"] = _pick(z, cut, g.uniform("u.draft", (n * B,)))
        s["uniforms"] = g.uniform("u", (n, B))
        i32 = dict(dtype=torch.int32, device=DEV)
        s["out"] = (torch.empty(n, **i32), torch.empty(n, **i32), torch.empty(n + 1, **i32),
                    torch.full((n * B,), -1, **i32))
    elif kind == "top":
        z = _logits(g, "logits", c["rows"], c["V"], "peaked", c["ld_extra"])
        s["logits"] = _cast(z, c["dtype"])[:, :c["V"]]
    else:
        n, B, P, V, K = c["n_seq"], c["B"], c["P"], c["V"], c["K"]
        z = _logits(g, "student", n * B, V, "peaked")
        # A student on its way to the teacher: near it, with errors of its own.
        t = z.view(n, B, V)[:, 1:P + 1].reshape(n * P, V) + g.normal("teacher", (n * P, V), 0.7)
        top = _top(t, min(K, V), c["temperature"])
        s["ids"] = top[0].view(n, P, -1).contiguous()
        s["values"] = top[1].view(n, P, -1).contiguous()
        s["rest"] = top[2].view(n, P).contiguous() if c["rest"] else None
        s["labels"] = g.ints("labels", (n, B - 1), V).to(torch.int32) if c["labels"] else None
        s["student"] = _cast(z, c["dtype"])
        s["alpha"] = 0.5
        s["grad_loss"] = torch.tensor([0.0, 0.0, 1.0], device=DEV)
    return s


# ------------------------------------------------------------------- the plain form

def _cut(z, settings):
    """The cut of every row: how many entries are kept, the last kept entry (-inf, -1 where
    every unmasked one is), the kept entries' log-sum-exp, and what the draws need."""
    T, top_k, top_p, min_p = settings
    z = z.float()
    V = z.shape[1]
    sv, si = torch.sort(z, dim=1, descending=True, stable=True)
    n_valid = (sv > NINF).sum(1, keepdim=True)
    m = sv[:, :1].to(F64)
    m = torch.where(n_valid > 0, m, torch.zeros_like(m))
    t = torch.where(T > 0, T, torch.ones_like(T))
    w = torch.exp((sv.to(F64) - m) / t)
    pos = torch.arange(V, device=z.device).unsqueeze(0)
    n_k = torch.where(top_k > 0, torch.minimum(top_k.long(), n_valid), n_valid)
    w = torch.where(pos < n_k, w, torch.zeros_like(w))
    cs = torch.cumsum(w, 1)
    n_p = 1 + (cs < top_p * cs[:, -1:]).sum(1, keepdim=True)
    n = torch.where(top_p < 1, torch.minimum(n_p, n_k), n_k)
    n_m = ((w >= min_p.clamp(max=1.0)) & (pos < n_k)).sum(1, keepdim=True)
    n = torch.where(min_p > 0, torch.minimum(n, n_m), n)
    n = torch.where(T > 0, n, n_valid.clamp(max=1))
    last = (n - 1).clamp(min=0)
    every = n == n_valid
    cut_logit = torch.where(every, torch.full_like(sv[:, :1], NINF), sv.gather(1, last))
    cut_index = torch.where(every, torch.full_like(last, -1), si.gather(1, last))
    lse = m / t + torch.log(torch.where(pos < n, w, torch.zeros_like(w)).sum(1, keepdim=True))
    lse = torch.where((T > 0) | (n == 0), lse, torch.zeros_like(lse))
    return dict(kept=n[:, 0].int(), cut_logit=cut_logit[:, 0], cut_index=cut_index[:, 0].int(),
                lse=lse[:, 0], T=t, greedy=T <= 0)


def _probs(z, cut, rows=slice(None)):
    """Truncated probabilities of whole rows."""
    z = z.float()
    idx = torch.arange(z.shape[1], device=z.device).unsqueeze(0)
    cl, ci = cut["cut_logit"][rows].unsqueeze(1), cut["cut_index"][rows].unsqueeze(1)
    keep = (z > cl) | ((z == cl) & (idx <= ci))
    p = torch.exp(z.to(F64) / cut["T"][rows] - cut["lse"][rows].unsqueeze(1))
    p = torch.where(cut["greedy"][rows], torch.ones_like(p), p)
    return torch.where(keep, p, torch.zeros_like(p))


def _inverse(w, u):
    """Lowest index whose running sum in index order passes u times the whole; -1 for no weight."""
    cs = torch.cumsum(w, 1)
    total = cs[:, -1:]
    i = (cs <= u.to(F64).unsqueeze(1) * total).sum(1, keepdim=True)
    idx = torch.arange(w.shape[1], device=w.device).unsqueeze(0)
    last = torch.where(w > 0, idx, torch.full_like(idx, -1)).amax(1, keepdim=True)
    return torch.minimum(i, last)[:, 0].int()


def _pick(z, cut, u):
    return _inverse(_probs(z, cut), u)


def _verify(s):
    c = s["case"]
    n, B, V = c["n_seq"], c["B"], c["V"]
    K = B - 1
    rows = _row_settings(s["settings"], n * B, B)
    tz = s["target_logits"].reshape(n * B, V)
    cut = _cut(tz, rows)
    p = _probs(tz, cut).view(n, B, V)
    kept, cl, ci, lse = s["draft_cut"]
    dcut = dict(kept=kept, cut_logit=cl, cut_index=ci, lse=lse, T=cut["T"], greedy=cut["greedy"])
    q = _probs(s["draft_logits"], dcut).view(n, B, V)[:, 1:]
    x = s["draft"].view(n, B)[:, 1:].long()
    px = p[:, :K].gather(2, x.unsqueeze(2)).squeeze(2)
    qx = q.gather(2, x.unsqueeze(2)).squeeze(2)
    ok = s["uniforms"][:, :K].to(F64) * qx < px
    n_acc = torch.cumprod(ok.long(), 1).sum(1)
    at = torch.arange(n, device=DEV)
    pn = p[at, n_acc]
    r = (pn - q[at, n_acc.clamp(max=K - 1)]).clamp(min=0)
    r = torch.where(((n_acc < K) & (r.sum(1) > 0)).unsqueeze(1), r, pn)
    nxt = _inverse(r, s["uniforms"][:, K]).long()
    slot = torch.arange(B, device=DEV).unsqueeze(0)
    commit = torch.cat([x, x[:, :1]], 1)
    commit = torch.where(slot == n_acc.unsqueeze(1), nxt.unsqueeze(1), commit)
    offs = torch.zeros(n + 1, dtype=torch.long, device=DEV)
    offs[1:] = torch.cumsum(n_acc + 1, 0)
    toks = torch.full((n * B + 1,), -1, dtype=torch.long, device=DEV)
    where = torch.where(slot <= n_acc.unsqueeze(1), offs[:n].unsqueeze(1) + slot, n * B)
    toks.scatter_(0, where.reshape(-1), commit.reshape(-1))
    return n_acc.int(), nxt.int(), offs.int(), toks[:n * B].int()


def _top(z, K, temperature):
    """The first K entries of every row's order, and the log-sum-exp of the others."""
    z = z.float()
    sv, si = torch.sort(z, dim=1, descending=True, stable=True)
    ids, values = si[:, :K].int(), sv[:, :K].contiguous()
    rest = torch.logsumexp(sv[:, K:].to(F64) / temperature, 1).float() if K < z.shape[1] else \
        torch.full((z.shape[0],), NINF, device=z.device)
    return ids, values, rest


def _distill(s):
    """Losses of every block, and the gradient of the sum L_CE + alpha L_KL.  The divergences are
    small differences of logarithms: they and what they are made of are taken in 64 bits."""
    c = s["case"]
    n, B, P, V, T = c["n_seq"], c["B"], c["P"], c["V"], c["temperature"]
    z = s["student"].float().view(n, B, V)
    t = s["values"].to(F64) / T
    if s["rest"] is not None:
        t = torch.cat([t, s["rest"].to(F64).unsqueeze(2)], 2)
    logp = t - torch.logsumexp(t, 2, keepdim=True)
    p = torch.exp(logp)
    zt = z[:, 1:P + 1].to(F64) / T
    m = zt.amax(2, keepdim=True)
    e = torch.exp(zt - m)
    q_sum = e.sum(2, keepdim=True)
    ids = s["ids"].long()
    K = ids.shape[2]
    logq = zt.gather(2, ids) - m - torch.log(q_sum)
    if s["rest"] is not None:
        q_rest = e.scatter(2, ids, 0.0).sum(2, keepdim=True)
        logq = torch.cat([logq, torch.log(q_rest) - torch.log(q_sum)], 2)
    kl = torch.where(p > 0, p * (logp - logq), torch.zeros_like(p)).sum(2)
    loss_kl = T * T / P * kl.sum() / n
    ce, loss_ce = None, torch.zeros((), dtype=F64, device=DEV)
    if s["labels"] is not None:
        lab = s["labels"].long().unsqueeze(2)
        z1 = z[:, 1:]
        ce = (torch.logsumexp(z1, 2, keepdim=True) - z1.gather(2, lab)).squeeze(2)
        loss_ce = ce.to(F64).mean()
    loss = torch.stack([loss_kl, loss_ce, loss_ce + s["alpha"] * loss_kl])
    out = [kl.float()] + ([ce] if ce is not None else []) + [loss.float()]
    if c["backward"]:
        grad = torch.zeros_like(z)
        q = e / q_sum
        if s["rest"] is not None:
            listed_ = q.gather(2, ids)
            q = (q * (1 - p[..., K:] * q_sum / q_rest)).scatter_(2, ids, listed_)
        q.scatter_add_(2, ids, -p[..., :K])
        grad[:, 1:P + 1] = (q * (s["alpha"] * T / (P * n))).float()
        if ce is not None:
            g1 = torch.softmax(z1, 2)
            g1.scatter_add_(2, lab, -torch.ones_like(lab, dtype=torch.float32))
            grad[:, 1:] += g1 / (n * (B - 1))
        out.append(grad.view(n * B, V).to(s["student"].dtype))
    return tuple(out)


def _plain(s):
    c = s["case"]
    if c["kind"] == "draw":
        cut = _cut(s["logits"], _row_settings(s["settings"], c["rows"], c["per"]))
        return (_pick(s["logits"], cut, s["uniforms"]), cut["kept"], cut["cut_logit"],
                cut["cut_index"], cut["lse"])
    if c["kind"] == "verify":
        return _verify(s)
    if c["kind"] == "top":
        return _top(s["logits"], c["K"], c["temperature"])
    return _distill(s)


# ------------------------------------------------------------------------------- a pass

def run(state):
    if not own:
        return _plain(state)
    from paper_2606_26744_amd import hdf
    s, c = state, state["case"]
    if c["kind"] == "draw":
        tokens, cut = hdf.sample_truncated(s["logits"], s["uniforms"], rows_per_seq=c["per"],
                                           **s["settings"])
        return (tokens, *cut)
    if c["kind"] == "verify":
        B, V = c["B"], c["V"]
        kept, cut_logit, cut_index, lse = s["draft_cut"]
        return hdf.accept_truncated(s["draft"][1:], s["draft_logits"][1:],
                                    (kept[1:], cut_logit[1:], cut_index[1:], lse[1:]),
                                    s["target_logits"], s["uniforms"], K=B - 1, draft_stride=B,
                                    ld=V, out=s["out"], **s["settings"])
    if c["kind"] == "top":
        return hdf.top_logits(s["logits"], c["K"], temperature=c["temperature"])
    kl, ce, loss, saved = hdf.distill_forward(s["student"], s["ids"], s["values"], s["rest"],
                                              s["labels"], B=c["B"], temperature=c["temperature"],
                                              alpha=s["alpha"])
    out = [kl] + ([ce] if ce is not None else []) + [loss]
    if c["backward"]:
        out.append(hdf.distill_backward(s["student"], s["ids"], s["labels"], saved, B=c["B"],
                                        temperature=c["temperature"], alpha=s["alpha"],
                                        grad_loss=s["grad_loss"]))
    return tuple(out)


def work(case):
    """Bytes that a pass reads and writes at the least (every logit of the rows that matter once,
    every output once) and its arithmetic (an exponential and a few sums a logit)."""
    c = case
    el = 2 if c["dtype"] == "bf16" else 4
    V = c["V"]
    if c["kind"] == "draw":
        return dict(bytes=c["rows"] * (V * el + 28), flops=4 * c["rows"] * V)
    if c["kind"] == "verify":
        rows = c["n_seq"] * c["B"]
        return dict(bytes=rows * (V * el + 40) + c["n_seq"] * V * 4,
                    flops=4 * rows * V + 6 * c["n_seq"] * V)
    if c["kind"] == "top":
        return dict(bytes=c["rows"] * (V * el + 8 * c["K"] + 4), flops=4 * c["rows"] * V)
    n, B = c["n_seq"], c["B"]
    rows = n * (B - 1) if c["labels"] else n * c["P"]
    b, f = rows * V * el + n * c["P"] * (8 * c["K"] + 8) + n * B * 8, 4 * rows * V
    if c["backward"]:
        b, f = b + n * B * V * el, f + 4 * rows * V
    return dict(bytes=b, flops=f)


# ------------------------------------------------------------------- 64-bit definitions

def _keys(z):
    """Integers in the order of the float values (z without -0)."""
    b = (z + 0.0).view(torch.int32).long()
    return torch.where(b >= 0, b, -(b & 0x7FFFFFFF))


def _bisect(keys, reached):
    """Per row the greatest key k for which reached(k) holds; reached(k) is monotone: it holds
    for the least key of all."""
    lo = torch.full_like(keys[:, :1], -0x7F800001)
    hi = torch.full_like(lo, 0x7F800001)
    while bool((hi - lo > 1).any()):
        mid = (lo + hi) // 2
        ok = reached(mid)
        lo, hi = torch.where(ok, mid, lo), torch.where(ok, hi, mid)
    return lo


def _exact_cut(z, settings):
    """The kept entries of every row as a mask, the last kept entry's key and index, weights."""
    T, top_k, top_p, min_p = settings
    z = z.float()
    rows, V = z.shape
    keys = _keys(z)
    valid = z > NINF
    idx = torch.arange(V, device=z.device).unsqueeze(0)
    m = z.amax(1, keepdim=True).to(F64)
    t = torch.where(T > 0, T, torch.ones_like(T))
    w = torch.where(valid, torch.exp((z.to(F64) - torch.where(m > NINF, m, 0.0)) / t), 0.0)

    def first(of, count, extra=None):
        """The first entries of the order until `of` sums to `count`, among those of `extra`."""
        have = of if extra is None else torch.where(extra, of, torch.zeros_like(of))
        total = have.sum(1, keepdim=True)
        count = torch.minimum(count, total)
        k = _bisect(keys, lambda q: torch.where(keys >= q, have, torch.zeros_like(have))
                    .sum(1, keepdim=True) >= count)
        above = torch.where(keys > k, have, torch.zeros_like(have)).sum(1, keepdim=True)
        tie = (keys == k) & (have > 0)
        run = above + torch.cumsum(torch.where(tie, have, torch.zeros_like(have)), 1)
        before = run - torch.where(tie, have, torch.zeros_like(have))
        return (keys > k) | (tie & (before < count))

    one = valid.to(F64)
    n_valid = one.sum(1, keepdim=True)
    keep = valid & ((top_k <= 0) | first(one, torch.where(top_k > 0, top_k, n_valid)))
    zk = torch.where(keep, w, 0.0).sum(1, keepdim=True)
    keep = keep & ((top_p >= 1) | first(w, top_p * zk, keep))
    keep = keep & ((min_p <= 0) | (w >= min_p.clamp(max=1.0)))
    best = _bisect(keys, lambda q: ((keys >= q) & valid).any(1, keepdim=True))
    lead = torch.where((keys == best) & valid, idx, V).amin(1, keepdim=True)
    keep = torch.where(T > 0, keep, (idx == lead) & valid)
    kept = keep.sum(1, keepdim=True)
    every = kept == n_valid
    low = torch.where(keep, z, float("inf")).amin(1, keepdim=True)
    at = torch.where(keep & (z == low), idx, -1).amax(1, keepdim=True)
    mass = torch.where(keep, w, 0.0)
    lse = torch.where(T > 0, m / t + torch.log(mass.sum(1, keepdim=True)), 0.0)
    lse = torch.where(kept > 0, lse, NINF)
    p = torch.where(T > 0, mass / mass.sum(1, keepdim=True), keep.to(F64))
    return dict(kept=kept[:, 0].int(), cut_logit=torch.where(every, NINF, low)[:, 0],
                cut_index=torch.where(every, -1, at)[:, 0].int(), lse=lse[:, 0],
                p=torch.where(kept > 0, p, 0.0))


def _exact_pick(p, u):
    total = p.sum(1, keepdim=True)
    passed = torch.cumsum(p, 1) > u.to(F64).unsqueeze(1) * total
    V = p.shape[1]
    idx = torch.arange(V, device=p.device).unsqueeze(0)
    first = torch.where(passed & (p > 0), idx, V).amin(1)
    last = torch.where(p > 0, idx, -1).amax(1)
    return torch.where(first < V, first, last).int()


def _exact_verify(s):
    c = s["case"]
    n, B, V = c["n_seq"], c["B"], c["V"]
    rows = _row_settings(s["settings"], n * B, B)
    p = _exact_cut(s["target_logits"].reshape(n * B, V), rows)["p"].view(n, B, V)
    q = _exact_cut(s["draft_logits"], rows)["p"].view(n, B, V)
    x = s["draft"].view(n, B).tolist()
    u = s["uniforms"].double().tolist()
    acc, nxt, offs, toks = [], [], [0], []
    for i in range(n):
        k = 0
        while k < B - 1 and u[i][k] * float(q[i, k + 1, x[i][k + 1]]) < float(p[i, k, x[i][k + 1]]):
            k += 1
        r = p[i, k]
        if k < B - 1:
            d = (p[i, k] - q[i, k + 1]).clamp(min=0)
            r = d if float(d.sum()) > 0 else r
        t = int(_exact_pick(r.unsqueeze(0), s["uniforms"][i:i + 1, B - 1])[0])
        acc.append(k)
        nxt.append(t)
        offs.append(offs[-1] + k + 1)
        toks += x[i][1:k + 1] + [t]
    toks += [-1] * (n * B - len(toks))
    return tuple(torch.tensor(v, dtype=torch.int32, device=DEV) for v in (acc, nxt, offs, toks))


def _exact_top(s):
    c = s["case"]
    z = s["logits"].float().cpu()
    order = torch.argsort(z.to(F64), dim=1, descending=True, stable=True)
    ids = order[:, :c["K"]]
    listed_ = torch.zeros_like(z, dtype=torch.bool).scatter_(1, ids, True)
    rest = torch.logsumexp((z.to(F64) / c["temperature"]).masked_fill(listed_, NINF), 1)
    return ids.int().to(DEV), z.gather(1, ids).to(F64).to(DEV), rest.to(DEV)


def _exact_distill(s):
    c = s["case"]
    n, B, P, V, T = c["n_seq"], c["B"], c["P"], c["V"], c["temperature"]
    z = s["student"].to(F64).view(n, B, V).requires_grad_(c["backward"])
    kls, ce = [], None
    for i in range(n):   # a block at a time, so that a full batch fits
        logq = torch.log_softmax(z[i, 1:P + 1] / T, 1)
        ids = s["ids"][i].long()
        t = s["values"][i].to(F64) / T
        lq = logq.gather(1, ids)
        if s["rest"] is not None:
            t = torch.cat([t, s["rest"][i].to(F64).unsqueeze(1)], 1)
            out = torch.logsumexp(logq.scatter(1, ids, NINF), 1, keepdim=True)
            lq = torch.cat([lq, out], 1)
        lp = torch.log_softmax(t, 1)
        kls.append((lp.exp() * (lp - lq)).sum(1))
    kl = torch.stack(kls)
    loss_kl = T * T / P * kl.sum() / n
    loss_ce = torch.zeros((), dtype=F64, device=DEV)
    if s["labels"] is not None:
        ce = -torch.log_softmax(z[:, 1:], 2).gather(2, s["labels"].long().unsqueeze(2)).squeeze(2)
        loss_ce = ce.mean()
    total = loss_ce + s["alpha"] * loss_kl
    loss = torch.stack([loss_kl, loss_ce, total])
    outs = [kl] + ([ce] if ce is not None else []) + [loss]
    res = [o.detach() for o in outs]
    if c["backward"]:
        res.append(torch.autograd.grad(total, z)[0].view(n * B, V))
    return tuple(res)


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["kind"] == "draw":
        if c["rows"] * c["V"] > 1 << 28:
            return None
        cut = _exact_cut(s["logits"], _row_settings(s["settings"], c["rows"], c["per"]))
        return (_exact_pick(cut["p"], s["uniforms"]), cut["kept"], cut["cut_logit"].to(F64),
                cut["cut_index"], cut["lse"])
    if c["kind"] == "verify":
        return _exact_verify(s)
    if c["kind"] == "top":
        return _exact_top(s)
    return _exact_distill(s)
