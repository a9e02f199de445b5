"""Batches without sequences: outputs that have entries all the same are written."""
import pytest
import torch

from paper_2606_26744_amd import hdf

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_losses_of_no_block():
    z = torch.empty(0, 50, device=DEV)
    ids, val = torch.empty(0, 2, 4, dtype=torch.int32, device=DEV), torch.empty(0, 2, 4, device=DEV)
    out = (torch.empty(0, 2, device=DEV), None, torch.full((3,), 7.0, device=DEV),
           torch.empty(4096, dtype=torch.uint8, device=DEV))
    loss = hdf.distill_forward(z, ids, val, B=3, out=out)[2]
    assert loss is out[2] and not loss.any()


@pytest.mark.parametrize("given", [True, False])
def test_commits_of_no_sequence(given):
    z, i = torch.empty(0, 50, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    cut = hdf.Truncation(i, torch.empty(0, device=DEV), i, torch.empty(0, dtype=torch.float64, device=DEV))
    out = tuple(torch.full((n,), 7, dtype=torch.int32, device=DEV) for n in (1, 1, 3, 1)) if given else None
    used = [torch.full((1,), 9, dtype=torch.int32, device=DEV) for _ in range(64)]
    del used   # so that a fresh tensor is not zero by chance
    acc, anc, offs, _ = hdf.accept_truncated(i, z, cut, torch.empty(0, 4, 50, device=DEV),
                                             torch.empty(0, 4, device=DEV), K=3, draft_stride=4, out=out)
    assert offs.tolist() == ([0, 7, 7] if given else [0])
    if given:
        hdf.accept_truncated(i, z, cut, torch.empty(0, 4, 50, device=DEV), torch.empty(0, 4, device=DEV),
                             K=3, draft_stride=4, out=(out[0], out[1], None, None))
