"""GPU tests of hdf.block_attention_kv4 with a bound of the contexts that its page table does not reach."""
import pytest
import torch

from paper_2606_26744_amd import hdf
from tests.test_gpu_kv4_attention import BF, F32, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hd,B,H", [(BF, 128, 16, 8), (BF, 64, 1, 4), (F32, 64, 5, 6)])
@pytest.mark.parametrize("max_ctx", [129, 1501, 8192])
def test_a_bound_beyond_the_table(dtype, hd, B, H, max_ctx):
    """max_ctx as a loop keeps it, tables as wide as the longest context needs (two pages)."""
    print(f"[kv4 tables] {dtype} hd={hd} B={B} max_ctx={max_ctx}", flush=True)
    c = Case([77, 128, 0, 1], B, H, 2, hd, dtype, seed=31)
    assert c.kw["page_table"].shape[1] == 2
    want, lse0 = hdf.block_attention_kv4(c.q, c.kv4, 0, **c.kw)
    c.check(want, lse0)
    out, lse = hdf.block_attention_kv4(c.q, c.kv4, 0, **dict(c.kw, max_ctx=max_ctx))
    assert torch.equal(out, want) and torch.equal(lse, lse0)


def test_contexts_end_with_the_table():
    """A context of more positions than its table has pages for counts what the table holds; a table
    of no pages leaves the block's own keys."""
    c = Case([200, 40], 3, 4, 2, 64, BF, seed=32)
    kw = dict(c.kw, page_table=c.kw["page_table"][:, :2].contiguous(), max_ctx=4096)
    out, lse = hdf.block_attention_kv4(c.q, c.kv4, 0, **kw)
    c.ctx, c.k[0], c.v[0] = [128, 40], c.k[0][:128], c.v[0][:128]
    c.check(out, lse)
    kw["page_table"] = kw["page_table"][:, :0].contiguous()
    out, lse = hdf.block_attention_kv4(c.q, c.kv4, 0, **kw)
    c.ctx, c.k, c.v = [0, 0], [x[:0] for x in c.k], [x[:0] for x in c.v]
    c.check(out, lse)
