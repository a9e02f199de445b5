"""The drafter step and the decode loop over a 4-bit cache (hdf_draft_block_kv4).  Block states are
checked against the oracle's block over what the GPU's cache stands for (read back in 32 bits, where
that is exact); the rows a call appends against the oracle's keys and values, which they are off by
a quantisation step at most (keys: the greatest of 32 dims / 3.5; values: the greatest of a head / 6,
a bfloat16's step more)."""
import dataclasses

import numpy as np
import pytest
import torch

import synth
from oracle.accept import accept as ref_accept
from oracle.drafter import Weights, block_forward, context_kv
from oracle.numerics import as_f64
from paper_2606_26744_amd import hdf
from paper_2606_26744_amd.decode import PagedDecoder
from paper_2606_26744_amd.step import StepBuffers, drafter_step
from tests._case import bits
from tests._tol import STATE_ABS, assert_bf16_state_close, assert_f32_rows_close

pytestmark = pytest.mark.gpu


def _handle(wl, w, max_pos):
    dr = wl.drafter
    return hdf.DrafterHandle(w, n_layers=dr.n_layers, d=dr.d, n_heads=dr.n_heads,
                             head_dim=dr.head_dim, d_ff=dr.d_ff, vocab=dr.vocab, eps=dr.eps,
                             rope_theta=dr.rope_theta, rope_max_pos=max_pos)


def _weights(wl, w):
    dr = wl.drafter
    wb = {k: ([bits(x) for x in v] if isinstance(v, list) else bits(v)) for k, v in w.items()}
    return Weights(wb, d=dr.d, n_layers=dr.n_layers, n_heads=dr.n_heads, head_dim=dr.head_dim,
                   d_ff=dr.d_ff, vocab=dr.vocab, eps=dr.eps, rope_theta=dr.rope_theta, dtype=wl.dtype)


def _read(kv4, layer, rows):
    n = rows.numel()
    k, v = hdf.kv4_read_rows(kv4, layer, n, rows=rows, dtype=torch.float32)
    return k.cpu().numpy().astype(np.float64), v.cpu().numpy().astype(np.float64)


def _check_appended(got, want, block, levels, what):
    """got within a step of want, of the greatest of `block` elements over `levels`."""
    n, d = want.shape
    top = np.abs(want).reshape(n, d // block, block).max(2)
    step = np.repeat(top, block, axis=1) / levels
    err = np.abs(got - want)
    assert (err <= 1.02 * step + 2 * STATE_ABS).all(), (what, float((err - step).max()))


def _check_hidden(wl, got, want, what):
    if wl.dtype == "bf16":
        assert_bf16_state_close(as_f64(got), want, what)
    else:
        assert_f32_rows_close(got, want, what)


def _workload(dtype, hd, B):
    wl = synth.small_bf16() if dtype == "bf16" else synth.tiny_fp32()
    if hd == 128:
        wl.drafter = synth.DrafterShape(d=512, n_layers=2, n_heads=4, head_dim=128, d_ff=1024, vocab=1000)
        wl.d = 512
    return dataclasses.replace(wl, block=B)


@pytest.mark.parametrize("dtype,hd,B,ctx,new,paged", [
    ("bf16", 128, 16, [300, 64, 17], [20, 5, 17], True),       # one launch for both projections
    ("bf16", 64, 5, [1, 63, 64, 130], [1, 7, 0, 130], False),  # a whole context among them
    ("bf16", 128, 20, [700, 90], [300, 60], True),             # rows of their own in the launch
    ("bf16", 128, 4, [2500, 8], [2500, 3], False),             # projected apart
    ("bf16", 64, 8, [500], [0], True),                         # nothing new
    ("f32", 64, 8, [200, 3], [60, 3], True),
    ("f32", 128, 3, [70], [70], False),
])
def test_block_over_a_4bit_cache(dtype, hd, B, ctx, new, paged):
    print(f"[kv4 drafter] {dtype} hd={hd} B={B} ctx={ctx} new={new} paged={paged}", flush=True)
    wl = dataclasses.replace(_workload(dtype, hd, B), n_seq=len(ctx), ctx_lens=list(ctx))
    dr = wl.drafter
    w = synth.drafter_weights(wl, device="cuda", random_norms=True)
    h = _handle(wl, w, max(ctx) + B)
    tiles = [(t + 63) // 64 for t in ctx]
    total = sum(tiles) + 3
    order = np.random.default_rng(5).permutation(total) if paged else np.arange(total)
    at = np.concatenate([[0], np.cumsum(tiles)])
    pages = [order[at[s]:at[s + 1]].tolist() for s in range(len(ctx))]
    kv4, none = h.alloc_kv(64 * total, kv_bits=4)
    assert none is None
    kv4.fill_(0xFF)
    kw = {}
    if paged:
        pt = np.full((len(ctx), max(tiles) + 1), -1, dtype=np.int32)
        for s, p in enumerate(pages):
            pt[s, :len(p)] = p
        kw["page_table"] = torch.from_numpy(pt).cuda()
    else:
        kw["kv_offsets"] = torch.tensor(hdf.kv_slot_offsets(ctx), dtype=torch.int32, device="cuda")
    rows = [hdf.paged_rows(pages[s], ctx[s], "cuda") for s in range(len(ctx))]
    for s, (T, n) in enumerate(zip(ctx, new)):
        for l in range(dr.n_layers):
            if T > n:
                k, v = synth.kv_prefix(wl, T - n, l, device="cuda", sub=s)
                hdf.kv4_write_rows(kv4, l, k, v, rows=rows[s][:T - n].contiguous())
    before = kv4.clone()
    no = [0]
    for n in new:
        no.append(no[-1] + n)
    y = synth.reduced_states(wl, no[-1], device="cuda")
    tokens = synth.block_tokens(wl, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    args = dict(ctx_len=torch.tensor(ctx, **i32), max_ctx=max(ctx), y_new=y,
                new_offsets=torch.tensor(no, **i32), kv_k=kv4, kv_vt=None, tokens=tokens, **kw)
    hidden = h.draft_block(**args)
    W = _weights(wl, w)
    for s, (T, n) in enumerate(zip(ctx, new)):
        ctx_kv = [_read(kv4, l, rows[s]) for l in range(dr.n_layers)]
        want = block_forward(W, ctx_kv, bits(tokens)[s])
        _check_hidden(wl, bits(hidden[s * B:(s + 1) * B]), want, f"hidden of {s}")
        fresh = context_kv(W, as_f64(bits(y[no[s]:no[s + 1]])), np.arange(T - n, T))
        for l in range(dr.n_layers):
            _check_appended(ctx_kv[l][0][T - n:], fresh[l][0], 32, 3.5, "keys")
            _check_appended(ctx_kv[l][1][T - n:], fresh[l][1], dr.head_dim, 6.0, "values")
            if T > n:
                prefix = rows[s][:T - n].contiguous()
                for a, b in zip(_read(kv4, l, prefix), _read(before, l, prefix)):
                    assert np.array_equal(a, b)
    # Again over the same cache, with a workspace of a larger call: the same states.
    ws = torch.full((h.workspace_bytes(len(ctx), B, no[-1] + 50, max(ctx), kv_bits=4),), 0xFF,
                    dtype=torch.uint8, device="cuda")
    assert torch.equal(h.draft_block(ws=ws, **args), hidden)


def test_a_prompt_longer_than_one_projection():
    """More new rows than one launch projects (16384): the keys and values of the last ones."""
    wl = dataclasses.replace(_workload("bf16", 64, 2), n_seq=1, ctx_lens=[16500])
    dr, T = wl.drafter, 16500
    w = synth.drafter_weights(wl, device="cuda", random_norms=True)
    h = _handle(wl, w, T + 2)
    kv4, _ = h.alloc_kv(64 * 260, kv_bits=4)
    i32 = dict(dtype=torch.int32, device="cuda")
    y = synth.reduced_states(wl, T, device="cuda")
    tokens = synth.block_tokens(wl, device="cuda")
    args = dict(ctx_len=torch.tensor([T], **i32), max_ctx=T, new_offsets=torch.tensor([0, T], **i32),
                kv_offsets=torch.tensor([0, 64 * 260], **i32), kv_k=kv4, kv_vt=None, tokens=tokens)
    hidden = h.draft_block(y_new=y, **args)
    assert torch.isfinite(hidden.float()).all()
    W = _weights(wl, w)
    at = np.r_[0:40, 16370:16400, 16480:16500]
    fresh = context_kv(W, as_f64(bits(y[torch.from_numpy(at).cuda()])), at)
    rows = torch.from_numpy(at.astype(np.int32)).cuda()
    for l in range(dr.n_layers):
        k, v = _read(kv4, l, rows)
        _check_appended(k, fresh[l][0], 32, 3.5, "keys")
        _check_appended(v, fresh[l][1], dr.head_dim, 6.0, "values")


def test_pages_outside_the_pool_are_not_written():
    """Page numbers whose rows lie beyond 32 bits too: nothing is written, nothing attended to."""
    wl = dataclasses.replace(_workload("bf16", 64, 4), n_seq=2, ctx_lens=[70, 5])
    w = synth.drafter_weights(wl, device="cuda")
    h = _handle(wl, w, 80)
    i32 = dict(dtype=torch.int32, device="cuda")
    y = synth.reduced_states(wl, 75, device="cuda")
    tokens = synth.block_tokens(wl, device="cuda")
    W = _weights(wl, w)
    for page in (1 << 26, (1 << 31) - 1, 3, -1, -(1 << 26)):
        kv4, _ = h.alloc_kv(3 * 64, kv_bits=4)
        table = torch.tensor([[2, page], [1, -1]], **i32)
        hidden = h.draft_block(ctx_len=torch.tensor([70, 5], **i32), max_ctx=70, y_new=y,
                               new_offsets=torch.tensor([0, 70, 75], **i32), page_table=table,
                               kv_k=kv4, kv_vt=None, tokens=tokens)
        assert not kv4[:, :, 0].any(), page
        for s, rows in ((0, range(128, 192)), (1, range(64, 69))):
            kv = [_read(kv4, l, torch.tensor(list(rows), **i32)) for l in range(h.L)]
            n = len(rows)
            want = block_forward(W, kv, bits(tokens)[s], pos_shift=(70, 5)[s] - n)
            _check_hidden(wl, bits(hidden[4 * s:4 * s + 4]), want, f"page {page}, sequence {s}")


def _targets(drafts):
    """Copies the first draft, then differs."""
    n, K = drafts.shape
    t = drafts.clone()
    t[:, 1:] = (t[:, 1:] + 1) % 50
    return torch.cat([t, torch.full((n, 1), 7, dtype=torch.int32, device=drafts.device)], 1).contiguous()


@pytest.mark.parametrize("chained", [False, True])
def test_decode_rounds_over_a_4bit_cache(chained):
    wl = _workload("bf16", 128, 8)
    prompts, rounds, B = [70, 5, 128], 4, 8
    wl = dataclasses.replace(wl, n_seq=3, ctx_lens=prompts)
    dr = wl.drafter
    w = synth.drafter_weights(wl, device="cuda")
    max_ctx = max(prompts) + (rounds + 1) * B
    h = _handle(wl, w, max_ctx + B)
    dec = PagedDecoder(h, 3, B, max_ctx, 20, sum(prompts), page_order=np.random.default_rng(1).permutation(20),
                       kv_bits=4)
    assert dec.kv_k.dtype == torch.uint8 and dec.kv_vt is None
    dec.set_anchors(torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda"))
    W = _weights(wl, w)
    red = synth.reducer_inputs(wl, sum(prompts), device="cuda", sub=50)
    out = dec.round(red["H"], prompts, red["W_g"], red["b_g"], _targets)
    counts = dec.next_counts(out["accept_len"])
    ctx = np.asarray(prompts, dtype=np.int64)
    if chained:
        dec.start_chain(counts)
    for r in range(rounds):
        ctx = ctx + counts
        if chained:
            H = synth.reducer_inputs(wl, 3 * B, device="cuda", sub=60 + r)["H"]
            out = dec.chained_round(H, red["W_g"], red["b_g"], _targets, record=True)
            tokens = out["tokens"]
            assert np.array_equal(out["ctx_len"].cpu().numpy(), ctx)
        else:
            H = synth.reducer_inputs(wl, int(counts.sum()), device="cuda", sub=60 + r)["H"]
            out = dec.round(H, counts, red["W_g"], red["b_g"], _targets)
            tokens = out["tokens"]
        torch.cuda.synchronize()
        for s in range(3):
            rows = hdf.paged_rows(dec.pages[s], int(ctx[s]), "cuda")
            kv = [_read(dec.kv_k, l, rows) for l in range(dr.n_layers)]
            assert np.isfinite(kv[0][0]).all() and np.abs(kv[0][0]).sum(1).all()
            want = block_forward(W, kv, bits(tokens)[s])
            _check_hidden(wl, bits(out["hidden"][s * B:(s + 1) * B]), want, f"round {r} sequence {s}")
        acc = ref_accept(out["drafts"].cpu().numpy(), out["targets"].cpu().numpy())[0]
        assert np.array_equal(out["accept_len"].cpu().numpy(), acc)
        counts = acc.astype(np.int64) + 1
    if chained:     # rows that no round committed are as they were
        ctx = dec.sync_lengths()
        for s in range(3):
            used = int(ctx[s]) - int(counts[s])
            tail = hdf.paged_rows(dec.pages[s], 64 * len(dec.pages[s]), "cuda")[used:].contiguous()
            for x in _read(dec.kv_k, 0, tail):
                assert not x.any()


def test_step_over_a_4bit_cache():
    """drafter_step takes the cache in the place of the keys."""
    wl = dataclasses.replace(_workload("bf16", 64, 4), n_seq=2, ctx_lens=[40, 9])
    w = synth.drafter_weights(wl, device="cuda")
    h = _handle(wl, w, 60)
    kv_k, kv_vt = h.alloc_kv(128, kv_bits=4)
    i32 = dict(dtype=torch.int32, device="cuda")
    red = synth.reducer_inputs(wl, 49, device="cuda")
    bufs = StepBuffers(h, 2, 4, 49, 40, wl.m, kv_bits=4)
    kw = dict(new_offsets=torch.tensor([0, 40, 49], **i32), ctx_len=torch.tensor([40, 9], **i32),
              max_ctx=40, kv_offsets=torch.tensor([0, 64, 128], **i32))
    tokens = synth.block_tokens(wl, device="cuda")
    targets = torch.zeros(2, 4, **i32)
    ws = bufs.ws.data_ptr()
    out = drafter_step(h, bufs, H_new=red["H"], W_g=red["W_g"], b_g=red["b_g"], kv_k=kv_k, kv_vt=kv_vt,
                       tokens=tokens, targets=targets, **kw)
    assert bufs.ws.data_ptr() == ws
    other = torch.zeros_like(kv_k)
    hidden = h.draft_block(y_new=out["Y"], kv_k=other, kv_vt=None, tokens=tokens, **kw)
    assert torch.equal(hidden, out["hidden"]) and torch.equal(other, kv_k)


def test_other_caches_are_refused():
    wl = _workload("bf16", 64, 4)
    h = _handle(wl, synth.drafter_weights(wl, device="cuda"), 60)
    kv4, _ = h.alloc_kv(64, kv_bits=4)
    i32 = dict(dtype=torch.int32, device="cuda")
    args = dict(ctx_len=torch.zeros(1, **i32), max_ctx=10, new_offsets=torch.zeros(2, **i32),
                y_new=torch.zeros(0, h.d, dtype=h.torch_dtype, device="cuda"),
                kv_offsets=torch.tensor([0, 64], **i32), tokens=torch.zeros(1, 4, **i32))
    for bad in (dict(kv_k=kv4, kv_vt=kv4), dict(kv_k=kv4[:0], kv_vt=None),
                dict(kv_k=hdf.kv4_alloc(h.L, h.nh + 1, h.hd, 64), kv_vt=None),
                dict(kv_k=h.alloc_kv(64)[0], kv_vt=None)):
        with pytest.raises(ValueError):
            h.draft_block(**args, **bad)
    with pytest.raises(ValueError):
        h.alloc_kv(64, kv_bits=8)
