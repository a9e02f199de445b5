"""What is left beside a row's top logits, where logits over the temperature are large or lie far
apart: the log-sum-exp of the unlisted entries whatever their distance from zero and from the listed.

Tolerance: a weight 2^a is off by |a| 2^-24 (its exponent, rounded once, weighs 0.54 at the most) and
an ulp of the instruction, 2^-23; a thread adds 32 in fp32, 31 * 2^-24 at the worst; the rest is
64-bit.  So the sum is right to (0.54 * 0.35 + 1 + 15.5) * 2^-23 < 2.0e-6, its logarithm absolutely,
and that is rounded to fp32 once."""
import numpy as np
import pytest
import torch

import test_gpu_truncation as base
from oracle import truncation as tr
from paper_2606_26744_amd import hdf

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _check(z, K, T):
    ids, values, rest = hdf.top_logits(z, K, temperature=T)
    torch.cuda.synchronize()
    zn = base._np(z)
    for r in range(z.shape[0]):
        i, v, s = tr.top_logits(zn[r], K, T)
        assert ids[r].tolist() == i.tolist() and base._np(values[r]).tolist() == v.tolist(), r
        got = float(rest[r])
        with np.errstate(over="ignore"):
            same = got == float(np.float32(s))
        assert same or abs(got - s) <= 2.0e-6 + 2.0 ** -24 * abs(s), (r, got, s)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1e-39, 1e-30, 1e-14, 1e-9, 1e-7, 1e-5, 1e-3, 1e3, 3e38])
@pytest.mark.parametrize("rows", [3, 300])
def test_any_temperature(rows, T, dtype):
    z = base._logits(rows, 9001, 7, dtype, "flat")
    z[1] = (z[1] * 2).round() / 2
    for K in (1, 20):
        _check(z[[0, 1, rows - 1]] if rows == 3 else z, K, T)


@pytest.mark.parametrize("scale", [1e-38, 1e6, 1e10, 1e30])
def test_any_scale(scale):
    z = base._logits(3, 20011, 8, kind="flat") * scale
    _check(z, 20, 1.0)
    _check(z, 20, scale)
    _check((z - z[:, 7:8]).clamp(max=0.0), 20, scale)   # relative to a logit of 0
    if scale < 1:
        _check((z - z.topk(21).values[:, 20:]) / 16, 20, 1e-39)
    z[:, ::3] += 100 * scale          # a list that is full of entries far above the others
    _check(z, 20, scale)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1.0, 0.25, 8.0])
@pytest.mark.parametrize("V", [3001, 30011])
def test_rest_of_the_lowest_value(V, T, dtype):
    """Masks by the type's lowest value: a list of all that is not masked, one more, one less."""
    z = base._logits(4, V, 9, dtype, "flat")
    low = torch.finfo(dtype).min
    live = torch.zeros(V, dtype=torch.bool, device=DEV)
    live[V // 50::V // 24] = True
    n = int(live.sum())
    z[:, ~live] = low
    z[1, :V // 2] = low                # chunks without a live entry
    z[2, ~live] = -1000.0
    z[3, ~live] = -1e30
    for K in (n - 1, n, n + 1, 100):
        _check(z, K, T)
