"""Nuclei that end among thousands of equal entries of little weight, which neither lists nor
histograms tell apart: the count of kept ones is that of the definition, by rational arithmetic.

A share p of the whole 1 + N w (one entry of weight 1, N of weight w) is reached with
ceil((p (1 + N w) - 1) / w) of the N.  Sums of about one round by 2^-53 some ten times, which is 2e-3
of an entry of weight 1e-12; weights are right to 1e-13 of themselves, 3e-8 of an entry of 250000.
The shares are chosen so that the quotient lies a fifth of an entry at least from a whole number."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2606_26744_amd import hdf

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _frac(x):
    return Fraction(float(np.float32(x)))


def _share(part, w, N):
    """fp32 share whose cut lies within the N near `part` of them, off the border; the quotient."""
    p = np.float32(float((1 + Fraction(part) * N * w) / (1 + N * w)))
    for _ in range(4000):
        x = (_frac(p) * (1 + N * w) - 1) / w
        if 0 < x < N and Fraction(1, 5) < x - math.floor(x) < Fraction(4, 5):
            return float(p), math.ceil(x)
        p = np.nextafter(p, np.float32(0))
    raise AssertionError("no share off the borders")


@pytest.mark.parametrize("rows", [2, 258])
@pytest.mark.parametrize("by", ["top_p", "top_k and top_p"])
@pytest.mark.parametrize("w,N,T", [(2e-10, 100000, 1.0), (1e-11, 200000, 1.0), (2e-10, 100000, 0.25),
                                   (3e-7, 30000, 1.0), (1e-12, 250000, 2.0)])
def test_cut_among_light_ties(w, N, T, by, rows):
    V = N + 1000
    low = np.float32(math.log(w) * T)
    # e^(low / T) by a series of 60 terms of its 64th part: exact to 1e-60 of itself.
    x = Fraction(float(low)) / _frac(T) / 64
    term, e = Fraction(1), Fraction(1)
    for i in range(1, 61):
        term = term * x / i
        term = Fraction(int(term * 10 ** 80), 10 ** 80)
        e += term
    wx = Fraction(1)
    for _ in range(64):
        wx = Fraction(int(wx * e * 10 ** 80), 10 ** 80)
    assert abs(float(wx) / math.exp(float(low) / T) - 1) < 1e-12
    z = torch.full((rows, V), -np.inf, device=DEV)
    z[:, 500:500 + N] = float(low)
    z[:, V - 1] = 0.0
    kw = dict(temperature=T)
    if by != "top_p":
        n_k = N - 777                     # further filter: the first N - 777 entries
        kw["top_k"] = n_k
        N = n_k - 1
    for part in (Fraction(1, 2), Fraction(1, 5)):
        p, light = _share(part, wx, N)
        # The draw: a third of the way through the light ones, between two of them.
        mass = 1 + light * wx
        u = np.float32(float((Fraction(light, 3) + Fraction(1, 2)) * wx / mass))
        at = math.floor(_frac(u) * mass / wx)
        off = _frac(u) * mass / wx - at
        tok, cut = hdf.sample_truncated(z, torch.full((rows,), float(u), device=DEV), top_p=p, **kw)
        for r in (0, rows - 1):
            assert int(cut.kept[r]) == 1 + light, (p, int(cut.kept[r]) - 1 - light)
            assert float(cut.cut_logit[r]) == low and int(cut.cut_index[r]) == 500 + light - 1
            if Fraction(1, 10) < off < Fraction(9, 10):
                assert int(tok[r]) == 500 + at


@pytest.mark.parametrize("rows", [2, 258])
def test_equal_light_entries_of_extreme_rows(rows):
    """The same where logits over the temperature pass fp32's range in between: at the least
    temperatures, and between logits whose difference is no fp32 value."""
    V = 40000
    big = float(torch.finfo(torch.float32).max)
    for low, top, T in ((-1e-37, 0.0, 1e-37), (-3e-38, 0.0, 1e-37), (-big, big, 1e38), (-big, big, 3e38)):
        w = math.exp((float(np.float32(low)) - float(np.float32(top))) / float(np.float32(T)))
        z = torch.full((rows, V), float(np.float32(low)), device=DEV)
        z[:, 77] = top
        p = float(np.float32(0.6))
        for kw, light in ((dict(), V - 1), (dict(top_k=V - 100), V - 101)):
            x = (p * (1 + light * w) - 1) / w
            assert 0.1 < x - math.floor(x) < 0.9
            _, cut = hdf.sample_truncated(z, torch.full((rows,), 0.5, device=DEV), temperature=T,
                                          top_p=p, **kw)
            for r in (0, rows - 1):
                assert int(cut.kept[r]) == 1 + math.ceil(x), (low, T, kw)
