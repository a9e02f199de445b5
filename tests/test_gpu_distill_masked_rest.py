"""Distillation where nothing outside a slot's list is left: every unlisted student logit masked, or
a list of the whole vocabulary.  The bucket then holds no student mass; a masked logit's gradient is
zero, however far the listed logits lie below zero.  Tolerances as in test_gpu_distill."""
import numpy as np
import pytest
import torch

import test_gpu_distill as base
from oracle import distill as od
from paper_2606_26744_amd import hdf

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _only_listed(dtype, T, at, labels, seed=3):
    """Slots whose student holds the listed tokens alone, about `at`; a bucket without mass."""
    n, B, P, K, V = 2, 5, 4, 12, 2503 if labels else 20011   # of one part, of three
    c = base._case(n, B, P, K, V, seed, dtype, labels=labels, T=T, ld=V + 2, offset=1)
    z = c["z"]
    g = torch.Generator().manual_seed(seed)
    for s in range(n):
        for k in range(1, P + 1):
            ids = c["ids"][s, k - 1].long()
            listed = (at + 2 * T * torch.randn(K, generator=g)).to(dtype).to(DEV)
            z[s * B + k] = -np.inf
            z[s * B + k, ids] = listed
            if labels:
                c["lab"][s, k - 1] = ids[k]
    c["rest"].fill_(-np.inf)
    return c, B


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("labels", [True, False])
@pytest.mark.parametrize("T,at", [(1.0, 3.0), (1.0, -100.0), (1.0, -1000.0), (2.0, -300.0),
                                  (0.1, -10.0), (0.01, -10.0)])
def test_every_unlisted_column_masked(dtype, labels, T, at):
    c, B = _only_listed(dtype, T, at, labels)
    _, _, _, d = base._check(c, B, T)
    masked = torch.isneginf(c["z"])
    assert masked.any() and not d[masked].any()
    if labels:
        c["lab"][0, 0] = -100
    base._check(c, B, T, g_loss=(1.0, 0.0, 0.0))
    base._check(c, B, T, g_loss=(0.0, 1.0, 0.0))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,at", [(1.0, -100.0), (1.0, -1000.0), (0.01, -10.0)])
def test_lists_of_the_whole_vocabulary(dtype, T, at):
    for V in (1, 9, 40, 300):
        c = base._case(1, 4, 3, V, V, V, dtype, T=T)
        c["z"].mul_(T).add_(at)
        assert torch.isneginf(c["rest"]).all()
        base._check(c, 4, T)


@pytest.mark.parametrize("T,at", [(1.0, 3.0), (1.0, -100.0), (1.0, -1000.0), (0.01, -10.0)])
def test_bucket_of_mass_over_masked_columns(T, at):
    """A bucket that the student gives nothing: the divergence is infinite, the gradients are finite:
    (q - p) / T of the listed tokens, zero elsewhere, softmax less one of a masked label."""
    for dtype in (torch.float32, torch.bfloat16):
        c, B = _only_listed(dtype, T, at, True)
        c["rest"][:] = c["val"][:, :, 0] / T
        n, P, K = c["ids"].shape
        V = c["z"].shape[1]
        masked = int(torch.isneginf(c["z"][1]).nonzero()[0])
        c["lab"][0, 0] = masked
        kl, ce, _, saved = hdf.distill_forward(c["z"], c["ids"], c["val"], c["rest"], c["lab"], B=B,
                                               temperature=T)
        assert torch.isposinf(kl).all() and torch.isposinf(ce[0, 0])
        d = hdf.distill_backward(c["z"], c["ids"], c["lab"], saved, B=B, temperature=T,
                                 grad_kl=torch.ones(n, P, device=DEV),
                                 grad_ce=torch.ones(n, B - 1, device=DEV))
        step = torch.finfo(dtype).eps / 2
        for s in range(n):
            for k in range(1, P + 1):
                z = base._np(c["z"][s * B + k])
                toks, p, _ = od.teacher(c["ids"][s, k - 1].tolist(), base._np(c["val"])[s, k - 1],
                                        float(c["rest"][s, k - 1]), V, float(np.float32(T)))
                q = od._softmax(z / float(np.float32(T)))
                want, mag = q / T, q / T
                want[toks] -= p / T
                mag[toks] += p / T
                _, g = od.slot_ce(z, int(c["lab"][s, k - 1]))
                want += g
                mag += np.abs(g)
                got = base._np(d[s * B + k])
                tol = base.GREL * mag * (1 + step) + step * np.abs(want) + 1e-37
                assert (np.abs(got - want) <= tol).all(), (s, k)
