"""The step under serving settings (drafter_step_truncated): its draws come from its own logits'
truncated distributions and its verification equals the oracle's on the same logits, drafts and
target logits (the slots' offsets and strides, the shared workspace)."""
import numpy as np
import pytest
import torch

import synth
from _case import DraftCase
from oracle import truncation as tr
from paper_2606_26744_amd import hdf
from paper_2606_26744_amd.step import (StepBuffers, TruncatedStepBuffers, drafter_step,
                                       drafter_step_truncated)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("target_dtype", [torch.float32, torch.bfloat16])
def test_truncated_step(target_dtype):
    wl = synth.small_bf16()
    ctx, new = [512] * 4, [16] * 4
    n_new = sum(new)
    red = synth.reducer_inputs(wl, n_new, device="cuda", sub=5)
    case = DraftCase(wl, ctx, new, random_norms=False, sub=5,
                     y_from=torch.empty((n_new, wl.d), dtype=red["H"].dtype, device="cuda"))
    n, B, V = len(ctx), case.B, wl.drafter.vocab
    bufs = StepBuffers(case.h, n, B, n_new, case.max_ctx, wl.m)
    tb = TruncatedStepBuffers(case.h, n, B)
    g = torch.Generator(device="cuda").manual_seed(1)
    kw = dict(H_new=red["H"], W_g=red["W_g"], b_g=red["b_g"], new_offsets=case.new_offsets,
              ctx_len=case.ctx_len, max_ctx=case.max_ctx, kv_offsets=case.kv_offsets,
              kv_k=case.kv_k, kv_vt=case.kv_vt, tokens=case.tokens)
    # Targets near the drafter's own logits, so that some drafts are accepted.
    own = drafter_step(case.h, bufs, targets=None, logits=True, **kw)["logits"].clone()
    tgt = 0.3 * torch.randn((n, B, V), generator=g, device="cuda")
    tgt[:, :B - 1] += own.view(n, B, V)[:, 1:]
    tgt = tgt.to(target_dtype)
    cuts = dict(temperature=torch.tensor([0.8, 1.0, 0.0, 0.6], device="cuda"),
                top_k=torch.tensor([0, 50, 0, 400], dtype=torch.int32, device="cuda"),
                top_p=torch.tensor([0.9, 1.0, 1.0, 0.95], device="cuda"),
                min_p=torch.tensor([0.0, 0.05, 0.0, 0.0], device="cuda"))
    u0 = torch.rand(n * B, generator=g, device="cuda")
    u1 = torch.rand(n, B, generator=g, device="cuda")
    out = drafter_step_truncated(case.h, bufs, tb, target_logits=tgt, draft_uniforms=u0,
                                 accept_uniforms=u1, **cuts, **kw)
    torch.cuda.synchronize()
    assert torch.equal(out["logits"], own)
    z, t = own.double().cpu().numpy(), tgt.double().cpu().numpy()
    tok = out["tokens"].tolist()
    offs = out["commit_offsets"].tolist()
    toks = out["commit_tokens"].tolist()
    for s in range(n):
        c = {k: v[s].item() for k, v in cuts.items()}
        q = [tr.truncate(z[s * B + k], **c) for k in range(B)]
        assert tok[s * B:(s + 1) * B] == [tr.inverse(q[k][4], float(u0[s * B + k])) for k in range(B)]
        assert out["truncation"].kept[s * B:(s + 1) * B].tolist() == [x[0] for x in q]
        p = np.array([tr.truncate(t[s, i], **c)[4] for i in range(B)])
        k, nxt, commit = tr.accept(tok[s * B + 1:(s + 1) * B], np.array([x[4] for x in q[1:]]), p,
                                   u1[s].tolist())
        assert (int(out["accept_len"][s]), int(out["next_anchor"][s])) == (k, nxt)
        assert toks[offs[s]:offs[s + 1]] == commit
