"""Gradients whose rows lie between the logits' own, in the same memory: no byte is shared."""
import pytest
import torch

import test_gpu_distill as base
from paper_2606_26744_amd import hdf

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("off,ld,ldd", [(1003, 2006, 2006), (-1003, 2006, 2006), (1003, 4013, 4013),
                                        (12 * 1003, 1003, 1005), (1003, 2006, 4012),
                                        (1003, 2006, 3009), (1002, 2006, 2006)])
def test_interleaved_rows(off, ld, ldd, dtype):
    n, B, V = 3, 4, 1003
    c = base._case(n, B, 3, 9, V, 3, dtype)
    buf = torch.full((13 * 4100 * 2,), 5.0, dtype=dtype, device=DEV)
    z = torch.as_strided(buf, (n * B, V), (ld, 1), 1003)
    d = torch.as_strided(buf, (n * B, V), (ldd, 1), 1003 + off)
    columns = [{first + r * stride + i for r in range(n * B) for i in range(V)}
               for first, stride in ((0, ld), (off, ldd))]
    if columns[0] & columns[1]:
        with pytest.raises(hdf.HdfError, match="share memory"):
            base._check({**c, "z": z}, B, d_logits=d)
        return
    z.copy_(c["z"])
    base._check({**c, "z": z}, B, d_logits=d)
    assert torch.equal(z, c["z"])
