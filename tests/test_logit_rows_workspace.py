"""Given workspaces of the calls on rows of logits."""
import pytest
import torch

from paper_2606_26744_amd import hdf


def test_strided_workspaces_are_refused():
    """The kernels would write over what lies between its elements."""
    z, ws = torch.zeros(2, 10), torch.zeros(4096, dtype=torch.uint8)
    for view in (ws[::2], ws.view(64, 64)[:, :32]):
        with pytest.raises(ValueError, match="contiguous"):
            hdf._scratch(view, 1024, z)
    assert hdf._scratch(ws, 1024, z) is ws
    assert hdf._scratch(ws[256:], 1024, z).data_ptr() == ws.data_ptr() + 256


def test_too_small_workspaces_are_replaced():
    z, ws = torch.zeros(2, 10), torch.zeros(100, dtype=torch.uint8)
    assert hdf._scratch(ws, 1024, z).numel() >= 1024
    assert hdf._scratch(None, 0, z).numel() >= 1
