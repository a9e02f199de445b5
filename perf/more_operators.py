"""A key/value cache held in 4 bits, as cases that can be timed and checked: its rows quantised as
they are written and read back, and the attention of blocks of queries over it.

Where `own` is false, run() computes a case with elementary torch operations on a plain packed
cache; where it is true it makes the library's calls on the library's cache.  listed() gives the
sizes that stand for the operators, draw() more of the same ranges; prepare() makes what a program
holds before the call, exact() the same outputs in 64 bits from the definitions.

The cache: an element is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign (e2m1), times a scale.
  keys    a scale 2^e for 32 consecutive dims of a row's head: the least e with amax <= 7 * 2^e
          (-125 <= e <= 125), amax the largest magnitude of the 32;
  values  a scale s for the head of a row: the least bfloat16 with amax <= 6 * s (s >= 2^-126).
An element becomes the nearest code of x / scale, ties to the even code, beyond 6 the 6.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
F64 = torch.float64
NINF = float("-inf")
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------------------ cases

def listed():
    return [
        # One sequence's newest position into the cache of a model with few heads of keys.
        dict(name="append_one", kind="write", n=1, heads=8, hd=128, dtype="bf16", tiles=40,
             place="list", pad=0),
        # What eight sequences committed in a round, scattered over their pages.
        dict(name="append_round", kind="write", n=40, heads=32, hd=128, dtype="bf16", tiles=256,
             place="list", pad=0),
        # A prompt of 16384 positions, keys and values as columns of one projection.
        dict(name="write_prompt", kind="write", n=16384, heads=32, hd=128, dtype="bf16", tiles=256,
             place="run", pad=4096),
        # An odd piece of a prompt in 32 bits, from an odd row on, smaller heads.
        dict(name="write_piece", kind="write", n=1777, heads=6, hd=64, dtype="f32", tiles=33,
             place="run", pad=0),
        # Rows of a few pages handed to another machine.
        dict(name="read_pages", kind="read", n=129, heads=32, hd=64, dtype="bf16", tiles=128,
             place="list"),
        # A whole layer's cache read back.
        dict(name="read_layer", kind="read", n=65536, heads=32, hd=128, dtype="bf16", tiles=1024,
             place="run"),
        # The next token of one short conversation: a launch's latency.
        dict(name="attend_token", kind="attend", n_seq=1, B=1, heads=32, kv_heads=8, hd=128,
             dtype="bf16", ctx_lo=700, ctx_hi=700, block="none", fused=False),
        # A draft block of eight sequences of 2048 positions.
        dict(name="attend_round", kind="attend", n_seq=8, B=16, heads=32, kv_heads=32, hd=128,
             dtype="bf16", ctx_lo=2048, ctx_hi=2048, block="full", fused=False),
        # Draft blocks of a full serving batch, contexts of 1024 to 16384 positions.
        dict(name="attend_ragged", kind="attend", n_seq=64, B=16, heads=32, kv_heads=32, hd=128,
             dtype="bf16", ctx_lo=1024, ctx_hi=16384, block="full", fused=False),
        # The next token over one very long document.
        dict(name="attend_long", kind="attend", n_seq=1, B=1, heads=32, kv_heads=8, hd=128,
             dtype="bf16", ctx_lo=131072, ctx_hi=131072, block="causal", fused=False),
        # A target model that verifies the drafts of sixteen sequences, blocks of different lengths.
        dict(name="attend_verify", kind="attend", n_seq=16, B=16, heads=32, kv_heads=8, hd=128,
             dtype="bf16", ctx_lo=512, ctx_hi=8192, block="causal_ragged", fused=True),
        # A small drafter in 32 bits.
        dict(name="attend_f32", kind="attend", n_seq=3, B=5, heads=6, kv_heads=6, hd=64,
             dtype="f32", ctx_lo=77, ctx_hi=1501, block="full", fused=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "write", "read", "attend", "attend", "attend"])
    hd = rng.choice([64, 128, 128])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("write", "read"):
        heads = rng.choice([1, 2, 5, 8, 12, 32])
        most = 16384 if kind == "write" else 32768
        n = _log_int(rng, 1, most * 32 * 128 // (heads * hd * (2 if dtype == "f32" else 1)) // 2)
        place = rng.choice(["run", "run", "list"])
        case = dict(kind=kind, n=n, heads=heads, hd=hd, dtype=dtype, place=place,
                    tiles=(n + 63) // 64 + rng.randint(1, 40))
        if kind == "write":
            case["pad"] = rng.choice([0, 0, 64, heads * hd])
        return case
    kv_heads = rng.choice([1, 2, 5, 8, 8, 32])
    group = 1 if kv_heads == 32 else rng.choice([1, 2, 4, 7, 8])
    n_seq = _log_int(rng, 1, 64)
    B = rng.choice([1, 1, 2, 5, 8, 15, 16, 16, 33])
    most = 131072 if n_seq == 1 else 16384
    most = min(most, 500000 * 32 * 128 // (n_seq * kv_heads * hd * max(1, group * B // 16)
                                           * (4 if dtype == "f32" else 1)))
    hi = _log_int(rng, 1, max(most, 2))
    return dict(kind=kind, n_seq=n_seq, B=B, heads=kv_heads * group, kv_heads=kv_heads, hd=hd,
                dtype=dtype, ctx_lo=rng.choice([hi, max(1, hi // 16), 1]), ctx_hi=hi,
                block=rng.choice(["none", "full", "full", "causal", "causal_ragged"]),
                fused=rng.random() < 0.3)


# ----------------------------------------------------------------------------- inputs

def _gen(seed, name, i=0):
    g = torch.Generator(device=DEV)
    k = 0
    for ch in name:
        k = (k * 131 + ord(ch)) % 1_000_003
    g.manual_seed((int(seed) * 1_000_003 + k * 1009 + i) & ((1 << 62) - 1))
    return g


def _cast(x, dtype):
    return x.to(torch.bfloat16) if dtype == "bf16" else x


def _kv_rows(seed, i, n, heads, hd, dtype):
    """Keys and values [n, heads, hd] as projections leave them: channels of the keys that stand
    out by a factor of a few, values of another size every row."""
    g = _gen(seed, "rows", i)
    c = _gen(seed, "channels")
    lift = torch.exp(0.7 * torch.randn(heads, hd, generator=c, device=DEV))
    k = torch.randn(n, heads, hd, generator=g, device=DEV).mul_(lift)
    size = torch.exp(0.3 * torch.randn(n, heads, 1, generator=g, device=DEV))
    v = torch.randn(n, heads, hd, generator=g, device=DEV).mul_(size)
    return _cast(k, dtype), _cast(v, dtype)


def _places(c, seed):
    """Cache rows of a write or a read: a run of rows from an odd one on, or a list of rows that
    holds short runs and single rows."""
    cap = 64 * c["tiles"]
    if c["place"] == "run":
        row0 = 0 if c["n"] % 64 == 0 else min(5, cap - c["n"])
        return row0, None
    g = _gen(seed, "places")
    run = 5                                  # rows of a sequence lie together
    starts = torch.randperm(cap // run, generator=g, device=DEV)[:(c["n"] + run - 1) // run] * run
    rows = (starts.unsqueeze(1) + torch.arange(run, device=DEV)).reshape(-1)[:c["n"]]
    return 0, rows.to(torch.int32).contiguous()


def _lengths(c, seed):
    g = torch.Generator().manual_seed(int(seed) * 7919 + 17)
    u = torch.rand(c["n_seq"], generator=g)
    ctx = (c["ctx_lo"] + u * (c["ctx_hi"] - c["ctx_lo"] + 1)).long().clamp(max=c["ctx_hi"])
    blk = torch.full((c["n_seq"],), c["B"])
    if c["block"] == "causal_ragged":
        blk = torch.randint(1, c["B"] + 1, (c["n_seq"],), generator=g)
    return ctx.tolist(), blk.tolist()


def _queries(c, seed, i, k):
    """Queries of sequence i [B, heads, hd]: noise with a part of some key of the context, so that
    a few keys carry much of the weight."""
    g = _gen(seed, "queries", i)
    B, H, n = c["B"], c["heads"], c["kv_heads"]
    q = torch.randn(B, H, c["hd"], generator=g, device=DEV)
    at = torch.randint(0, k.shape[0], (B,), generator=g, device=DEV)
    near = k[at].float().unsqueeze(2).expand(B, n, H // n, c["hd"]).reshape(B, H, c["hd"])
    return _cast(q + 0.3 * near, c["dtype"])


def _attend_inputs(c, seed):
    """Per sequence: keys and values of the context, queries, keys and values of the block."""
    ctx, blk = _lengths(c, seed)
    for i, T in enumerate(ctx):
        k, v = _kv_rows(seed, i, T + c["B"], c["kv_heads"], c["hd"], c["dtype"])
        yield i, T, blk[i], k[:T], v[:T], _queries(c, seed, i, k), k[T:], v[T:]


def prepare(case, seed):
    c = case
    s = dict(case=c)
    if c["kind"] in ("write", "read"):
        n, heads, hd = c["n"], c["heads"], c["hd"]
        s["row0"], s["rows"] = _places(c, seed)
        k, v = _kv_rows(seed, 0, n, heads, hd, c["dtype"])
        if c["kind"] == "write":
            both = torch.zeros(n, 2 * heads * hd + c["pad"], dtype=k.dtype, device=DEV)
            s["k"], s["v"] = both[:, :heads * hd], both[:, heads * hd:2 * heads * hd]
            s["k"].copy_(k.view(n, -1))
            s["v"].copy_(v.view(n, -1))
        if own:
            from paper_2606_26744_amd import hdf
            s["kv4"] = hdf.kv4_alloc(1, heads, hd, 64 * c["tiles"])
            if c["kind"] == "read":
                hdf.kv4_write_rows(s["kv4"], 0, k.view(n, -1), v.view(n, -1), row0=s["row0"],
                                   rows=s["rows"])
        else:
            s["cache"] = _empty(64 * c["tiles"], heads, hd)
            if c["kind"] == "read":
                _store(s["cache"], _index(s, n), k, v)
        return s
    n_seq, B, H, n, hd = c["n_seq"], c["B"], c["heads"], c["kv_heads"], c["hd"]
    ctx, blk = _lengths(c, seed)
    max_pages = (max(ctx) + 63) // 64
    pages = sum((T + 63) // 64 for T in ctx) + 3
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(int(seed) + 5))
    table = torch.full((n_seq, max_pages), -1, dtype=torch.int32)
    at = 0
    for i, T in enumerate(ctx):
        m = (T + 63) // 64
        table[i, :m] = order[at:at + m].int()
        at += m
    s.update(ctx=ctx, blk=blk, max_ctx=c["ctx_hi"], page_table=table.to(DEV),
             ctx_len=torch.tensor(ctx, dtype=torch.int32, device=DEV),
             block_len=torch.tensor(blk, dtype=torch.int32, device=DEV)
             if c["block"] == "causal_ragged" else None)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    # Queries, keys and values of the block: columns of one projection, or tensors of their own.
    wide = (H + 2 * n) * hd
    qkv = torch.empty(n_seq, B, wide, dtype=dt, device=DEV)
    cols = (qkv[..., :H * hd], qkv[..., H * hd:(H + n) * hd], qkv[..., (H + n) * hd:])
    if own:
        from paper_2606_26744_amd import hdf
        s["kv4"] = hdf.kv4_alloc(1, n, hd, 64 * pages)
    else:
        s["cache"] = _empty(64 * pages, n, hd)
    for i, T, _, k, v, q, kb, vb in _attend_inputs(c, seed):
        rows = _sequence_rows(s, i, T)
        if own:
            hdf.kv4_write_rows(s["kv4"], 0, k.reshape(T, -1), v.reshape(T, -1), rows=rows.int())
        else:
            _store(s["cache"], rows, k, v)
        for col, x in zip(cols, (q, kb, vb)):
            col[i].copy_(x.reshape(B, -1))
    parts = [x if c["fused"] else x.contiguous() for x in cols]
    s["q"] = parts[0].view(n_seq, B, H, hd)
    s["kb"], s["vb"] = (parts[1].view(n_seq, B, n, hd), parts[2].view(n_seq, B, n, hd)) \
        if c["block"] != "none" else (None, None)
    # Outputs of slots behind a block's length stay as they are.
    s["out"] = (torch.zeros(n_seq, B, H, hd, dtype=dt, device=DEV),
                torch.zeros(n_seq, B, H, dtype=torch.float32, device=DEV))
    return s


# ------------------------------------------------------------------- the plain form

def _empty(cap, heads, hd):
    """Plain packed cache: two codes a byte, the scales' exponents, the values' scales."""
    u8 = dict(dtype=torch.uint8, device=DEV)
    return dict(k=torch.zeros(cap, heads, hd // 2, **u8), e=torch.zeros(cap, heads, hd // 32, **u8),
                v=torch.zeros(cap, heads, hd // 2, **u8),
                s=torch.zeros(cap, heads, 1, dtype=torch.bfloat16, device=DEV))


def _power(e):
    """2^e of whole numbers from their bits."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _codes(x, unit):
    """Codes of x / unit, packed; unit has few enough bits that its products here are exact."""
    a = x.abs()
    c = torch.zeros_like(a, dtype=torch.uint8)
    for i, t in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        c += (a > t * unit) if i % 2 == 0 else (a >= t * unit)
    c += torch.signbit(x).to(torch.uint8) * 8
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _store(cache, rows, k, v):
    rows = rows.long()
    n, heads, hd = k.shape
    x = k.float().view(n, heads, hd // 32, 32)
    m, e = torch.frexp(x.abs().amax(3, keepdim=True))
    e = torch.where(m <= 0.875, e - 3, e - 2).clamp(-125, 125)
    cache["k"][rows] = _codes(x, _power(e)).view(n, heads, hd // 2)
    cache["e"][rows] = (e + 127).to(torch.uint8).view(n, heads, hd // 32)
    x = v.float()
    amax = x.abs().amax(2, keepdim=True)
    s = ((amax / 6).view(torch.int32) & -65536).clamp(min=0x00800000)
    for _ in range(2):
        s = torch.where(6 * s.view(torch.float32) < amax, s + 65536, s)
    s = s.view(torch.float32)
    cache["v"][rows] = _codes(x, s)
    cache["s"][rows] = s.to(torch.bfloat16)


def _unpack(p):
    table = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device=DEV)
    c = torch.stack([p & 15, p >> 4], -1).flatten(-2)
    return table[c.int()]


def _load(cache, rows):
    """Keys and values of cache rows, in 32 bits."""
    rows = rows.long()
    k, v = _unpack(cache["k"][rows]), _unpack(cache["v"][rows])
    n, heads, hd = k.shape
    unit = _power(cache["e"][rows].to(torch.int32) - 127)
    k = (k.view(n, heads, hd // 32, 32) * unit.unsqueeze(3)).view(n, heads, hd)
    return k, v * cache["s"][rows].float()


def _index(s, n):
    if s["rows"] is not None:
        return s["rows"]
    return torch.arange(s["row0"], s["row0"] + n, device=DEV)


def _sequence_rows(s, i, T):
    t = torch.arange(T, device=DEV)
    return s["page_table"][i].long()[t // 64] * 64 + t % 64


def _plain(s):
    c = s["case"]
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    if c["kind"] in ("write", "read"):
        n, heads, hd = c["n"], c["heads"], c["hd"]
        rows = _index(s, n)
        if c["kind"] == "write":
            _store(s["cache"], rows, s["k"].reshape(n, heads, hd), s["v"].reshape(n, heads, hd))
        k, v = _load(s["cache"], rows)
        return k.view(n, -1).to(dt), v.view(n, -1).to(dt)
    out, lse = s["out"]
    B, H, n, hd = c["B"], c["heads"], c["kv_heads"], c["hd"]
    G = H // n
    for i, T in enumerate(s["ctx"]):
        b = s["blk"][i]
        k, v = _load(s["cache"], _sequence_rows(s, i, T))
        if s["kb"] is not None:
            k = torch.cat([k, s["kb"][i, :b].float()])
            v = torch.cat([v, s["vb"][i, :b].float()])
        q = s["q"][i, :b].float().view(b, n, G, hd).permute(1, 0, 2, 3).reshape(n, b * G, hd)
        x = torch.bmm(q, k.permute(1, 2, 0).contiguous()) * (1.0 / math.sqrt(hd))
        if c["block"].startswith("causal"):
            hide = torch.ones(b, b, dtype=torch.bool, device=DEV).triu(1)
            x[:, :, T:] = x[:, :, T:].masked_fill(hide.repeat_interleave(G, 0), NINF)
        m = x.amax(2, keepdim=True)
        p = torch.exp(x - m)
        total = p.sum(2, keepdim=True)
        o = torch.bmm(p, v.permute(1, 0, 2).contiguous()) / total
        out[i, :b] = o.view(n, b, G, hd).permute(1, 0, 2, 3).reshape(b, H, hd).to(dt)
        l = (m + torch.log(total)).view(n, b, G)
        lse[i, :b] = l.permute(1, 0, 2).reshape(b, H)
    return out, lse


# ------------------------------------------------------------------------------- a pass

def run(state):
    if not own:
        return _plain(state)
    from paper_2606_26744_amd import hdf
    s, c = state, state["case"]
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    if c["kind"] in ("write", "read"):
        if c["kind"] == "write":
            hdf.kv4_write_rows(s["kv4"], 0, s["k"], s["v"], row0=s["row0"], rows=s["rows"])
        return hdf.kv4_read_rows(s["kv4"], 0, c["n"], row0=s["row0"], rows=s["rows"], dtype=dt)
    return hdf.block_attention_kv4(s["q"], s["kv4"], 0, ctx_len=s["ctx_len"], max_ctx=s["max_ctx"],
                                   page_table=s["page_table"], k_blk=s["kb"], v_blk=s["vb"],
                                   block_len=s["block_len"],
                                   causal=c["block"].startswith("causal"), out=s["out"])


def work(case):
    """Bytes that a pass reads and writes at the least, and its arithmetic.  A key takes 4.25 bits
    an element, a value 4 and 16 bits a head."""
    c = case
    el = 2 if c["dtype"] == "bf16" else 4
    hd = c["hd"]
    row = 2 * (hd // 2) + hd // 32 + 2          # bytes of a position of one head in the cache
    if c["kind"] in ("write", "read"):
        cells = c["n"] * c["heads"]
        rows = 2 * cells * hd * el
        return dict(bytes=cells * row + rows * (2 if c["kind"] == "write" else 1),
                    flops=4 * cells * hd)
    keys = c["n_seq"] * (c["ctx_lo"] + c["ctx_hi"]) // 2
    slots = c["n_seq"] * c["B"]
    blocks = 2 * slots * c["kv_heads"] * hd * el if c["block"] != "none" else 0
    return dict(bytes=keys * c["kv_heads"] * row + 2 * slots * c["heads"] * hd * el + blocks,
                flops=4 * keys * c["B"] * c["heads"] * hd)


# ------------------------------------------------------------------- 64-bit definitions

def _nearest(y):
    """The level nearest to y, ties to the even place in the list, 6 beyond it."""
    levels = torch.tensor(LEVELS, dtype=F64, device=DEV)
    a = y.abs().clamp(max=6.0)
    hi = torch.searchsorted(levels, a).clamp(1, 7)
    up, down = levels[hi] - a, a - levels[hi - 1]
    take = (up < down) | ((up == down) & (hi % 2 == 0))
    return torch.where(take, levels[hi], levels[hi - 1]) * torch.sign(y)


def _exact_rows(k, v):
    """What the cache stands for."""
    n, heads, hd = k.shape
    x = k.to(F64).view(n, heads, hd // 32, 32)
    amax = x.abs().amax(3, keepdim=True)
    e = torch.floor(torch.log2(amax.clamp(min=2.0 ** -130))) - 4
    for _ in range(4):
        e = torch.where(7 * torch.exp2(e) < amax, e + 1, e)
    unit = torch.exp2(e.clamp(-125, 125))
    kd = (_nearest(x / unit) * unit).view(n, heads, hd)
    x = v.to(F64)
    need = (x.abs().amax(2, keepdim=True) / 6).clamp(min=2.0 ** -126)
    grid = torch.exp2(torch.floor(torch.log2(need)) - 7)
    s = torch.ceil(need / grid) * grid
    return kd, _nearest(x / s) * s


def exact(case, seed):
    c = case
    if c["kind"] in ("write", "read"):
        k, v = _kv_rows(seed, 0, c["n"], c["heads"], c["hd"], c["dtype"])
        kd = torch.empty(k.shape, dtype=F64, device=DEV)
        vd = torch.empty_like(kd)
        for a in range(0, c["n"], 4096):
            kd[a:a + 4096], vd[a:a + 4096] = _exact_rows(k[a:a + 4096], v[a:a + 4096])
        return kd.view(c["n"], -1), vd.view(c["n"], -1)
    B, H, n, hd = c["B"], c["heads"], c["kv_heads"], c["hd"]
    out = torch.zeros(c["n_seq"], B, H, hd, dtype=F64, device=DEV)
    lse = torch.zeros(c["n_seq"], B, H, dtype=F64, device=DEV)
    for i, T, b, k, v, q, kb, vb in _attend_inputs(c, seed):
        q = q[:b].to(F64)
        for h in range(n):                      # a head of keys at a time
            kd, vd = _exact_rows(k[:, h:h + 1], v[:, h:h + 1])
            kd, vd = kd[:, 0], vd[:, 0]
            if c["block"] != "none":
                kd = torch.cat([kd, kb[:b, h].to(F64)])
                vd = torch.cat([vd, vb[:b, h].to(F64)])
            for j in range(h * (H // n), (h + 1) * (H // n)):
                x = torch.mv(kd, q[0, j]).unsqueeze(0) if b == 1 else q[:, j] @ kd.t()
                x = x / math.sqrt(hd)
                if c["block"].startswith("causal"):
                    for a in range(b):
                        x[a, T + a + 1:] = NINF
                lse[i, :b, j] = torch.logsumexp(x, 1)
                out[i, :b, j] = torch.softmax(x, 1) @ vd
    return out, lse
