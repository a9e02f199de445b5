"""Distillation against the bounds of the sums as the kernels form them.

An exponent a (base 2) is off by 2^-24 |a| from its one rounding (two where logits are far from zero) and
2^-24 |a| from log2(e) / T in fp32, which weighs a term 2^a by |a| 2^a <= 0.54, and the instruction by
an ulp, 2^-23.  At most 15 fp32 additions in a row follow (7 of a vector's eight, 2 of four vectors, 6
over a wave; 3 + 3 + 6 of fp32 logits), 15 * 2^-24; the rest is 64-bit.  A sum is thus right to
(0.54 * 0.7 * 1.5 + 1 + 7.5) * 2^-23 < 1.1e-6, its logarithm to the same absolutely.  The bounds of
the losses follow from that as in test_gpu_distill.  A part of a gradient holds two such sums, four
roundings, and its own exponent's error: 2^-23 of the octaves between its logit and the greatest."""
import pytest
import torch

import test_gpu_distill as base

pytestmark = pytest.mark.gpu
REL = 1.1e-6


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rest,T", [(True, 1.0), (True, 2.0), (False, 1.0), (True, 0.5), (False, 3.0)])
@pytest.mark.parametrize("n,B,P,K,V", [(3, 6, 3, 20, 9001), (1, 4, 3, 128, 40009), (40, 2, 1, 5, 300),
                                       (1, 2, 1, 50, 151937), (2, 3, 2, 700, 2003)])
def test_losses_and_gradients(n, B, P, K, V, rest, T, dtype, monkeypatch):
    monkeypatch.setattr(base, "REL", REL)
    for labels in (True, False):
        c = base._case(n, B, P, K, V, V + K, dtype, rest, labels, T, ld=V + 3, offset=1)
        octaves = float(c["z"].max() - c["z"].min()) / min(T, 1.0) * 1.4427
        monkeypatch.setattr(base, "GREL", 2 * REL + (4 + 0.7 * octaves) * 2.0 ** -23)
        base._check(c, B, T)
