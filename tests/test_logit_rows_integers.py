"""Integers that the C calls hold in 32 bits: what does not fit is refused by name, not cut to its low
bits (a row count a sequence of 2^32 + 1 would read settings past their end)."""
import pytest
import torch

from paper_2606_26744_amd import hdf

Z = torch.zeros(4, 10)
INT = torch.zeros(4, dtype=torch.int32)
CUT = (INT, Z[:, 0].contiguous(), INT, Z[:, 0].double())


@pytest.mark.parametrize("value", [1 << 31, (1 << 32) + 1, 1 << 64])
def test_settings(value):
    with pytest.raises(ValueError, match="rows_per_seq"):
        hdf.sample_truncated(Z, rows_per_seq=value)
    for kw, what in ((dict(draft_stride=4, top_k=value), "top_k"), (dict(draft_stride=value), "draft_stride")):
        with pytest.raises(ValueError, match=what):
            hdf.accept_truncated(INT, Z, CUT, Z.view(1, 4, 10), Z, K=3, **kw)
    with pytest.raises(ValueError, match="top_k"):
        hdf.sample_truncated(Z, top_k=value)
    with pytest.raises(ValueError, match="K must"):
        hdf.top_logits(Z, value)


def test_rows_and_columns():
    for shape in ((1, (1 << 32) + 10), ((1 << 32) + 10, 1)):
        with pytest.raises(ValueError, match="rows and columns"):
            hdf.top_logits(torch.empty(shape, device="meta"), 3)


def test_the_greatest_that_fit():
    with pytest.raises(ValueError, match="device tensors"):
        hdf.sample_truncated(Z, top_k=(1 << 31) - 1, rows_per_seq=(1 << 31) - 1)
