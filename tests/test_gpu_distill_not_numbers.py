"""Distillation with logits that are no numbers: they reach their slot's losses and gradients, of
either type, and no other slot."""
import pytest
import torch

import test_gpu_distill as base
from paper_2606_26744_amd import hdf

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _nan(bits):
    return torch.tensor([bits], dtype=torch.int64).to(torch.int32).view(torch.float32).to(DEV)


def _grad(c, B, **kw):
    kl, ce, loss, saved = hdf.distill_forward(c["z"], c["ids"], c["val"], c["rest"], c["lab"], B=B)
    return kl, hdf.distill_backward(c["z"], c["ids"], c["lab"], saved, B=B, **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [0x7FC00000, 0x7FFFFFFF, 0xFFFFFFFF, 0xFFFF8000, 0x7FFF7FFF])
def test_nans_of_any_bits(bits, dtype):
    """A NaN from memory filled with ones stays one where it is rounded to 16 bits."""
    n, B, P, V = 2, 4, 3, 701
    for where in ("val", "rest", "kl"):
        c = base._case(n, B, P, 6, V, 4, dtype)
        g_kl = torch.ones(n, P, device=DEV)
        (c["val"][1, 1, 2:3] if where == "val" else c["rest"][1, 1:2] if where == "rest" else
         g_kl[1, 1:2]).copy_(_nan(bits))
        kl, d = _grad(c, B, grad_kl=g_kl)
        assert torch.isnan(kl).view(-1).tolist() == [where != "kl" and i == 4 for i in range(n * P)]
        assert torch.isnan(d[B + 2]).all(), where
        others = [r for r in range(n * B) if r != B + 2]
        assert torch.isfinite(d[others]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("where", ["student listed", "student unlisted", "teacher"])
def test_a_slot_with_one_is_not_a_number_throughout(where, value, rest, dtype):
    n, B, P, V = 2, 4, 3, 701
    c = base._case(n, B, P, 6, V, 5, dtype, rest=rest)
    if where == "teacher":
        c["val"][1, 1, 2] = value
    else:
        ids = c["ids"][1, 1].tolist()
        c["z"][B + 2, ids[3] if where == "student listed" else
               next(i for i in range(V) if i not in ids)] = value
    kl, d = _grad(c, B, grad_kl=torch.ones(n, P, device=DEV))
    assert torch.isnan(kl).view(-1).tolist() == [i == 4 for i in range(n * P)]
    assert torch.isnan(d[B + 2]).all()
    others = [r for r in range(n * B) if r != B + 2]
    assert torch.isfinite(d[others]).all()
