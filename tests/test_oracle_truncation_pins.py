"""The truncation oracle against cases worked out by hand, and its verification against the
distribution that it has to preserve."""
import numpy as np
import pytest

from oracle import truncation as tr

LOG = np.log


def test_cuts_by_hand():
    z = LOG(np.array([0.1, 0.4, 0.2, 0.3]))
    n, cl, ci, lse, p = tr.truncate(z, top_k=2)
    assert (n, ci) == (2, 3) and cl == z[3]
    np.testing.assert_allclose(p, [0, 4 / 7, 0, 3 / 7])
    np.testing.assert_allclose(lse, LOG(0.7))
    assert tr.truncate(z, top_p=0.39)[0] == 1
    assert tr.truncate(z, top_p=0.41)[0] == 2
    assert tr.truncate(z, top_p=0.71)[0] == 3
    assert tr.truncate(z, top_p=0.0)[0] == 1
    assert tr.truncate(z, min_p=0.49)[0] == 3         # 0.2 / 0.4 >= 0.49
    assert tr.truncate(z, min_p=1.0)[0] == 1
    # top_p counts the mass of the top_k entries: 0.4 / 0.7 >= 0.55 with one entry
    assert tr.truncate(z, top_k=2, top_p=0.55)[0] == 1
    assert tr.truncate(z, temperature=0.0)[4].tolist() == [0, 1, 0, 0]
    # T = 2 flattens: sqrt weights 0.316 0.632 0.447 0.548, whole 1.944
    assert tr.truncate(z, temperature=2.0, top_p=0.6)[0] == 2
    assert tr.truncate(z, temperature=2.0, top_p=0.61)[0] == 3


def test_ties_masks_and_whole_rows():
    z = np.array([1.0, 3.0, 3.0, -np.inf, 3.0, np.nan])
    assert tr.order(z).tolist() == [1, 2, 4, 0]
    assert tr.truncate(z, top_k=2)[:3] == (2, 3.0, 2)
    assert tr.truncate(z, min_p=1.0)[:3] == (3, 3.0, 4)
    assert tr.truncate(z, top_k=9)[:3] == (4, -np.inf, -1)
    n, cl, ci, lse, p = tr.truncate(np.full(3, -np.inf), top_k=1)
    assert (n, ci, lse) == (0, -1, -np.inf) and not p.any()
    assert tr.inverse(p, 0.5) == -1


def test_inverse_by_hand():
    p = np.array([0.0, 0.25, 0.0, 0.5, 0.25, 0.0])
    assert [tr.inverse(p, u) for u in (0.0, 0.249, 0.25, 0.749, 0.75, 1.0)] == [1, 1, 3, 3, 4, 4]


def test_top_logits_by_hand():
    ids, v, rest = tr.top_logits(np.array([0.0, 2.0, -np.inf, 2.0, 1.0]), 2, 2.0)
    assert ids.tolist() == [1, 3] and v.tolist() == [2.0, 2.0]
    np.testing.assert_allclose(rest, LOG(1 + np.exp(0.5)))
    ids, v, rest = tr.top_logits(np.array([0.0, -np.inf]), 3)
    assert ids.tolist() == [0, -1, -1] and rest == -np.inf


@pytest.mark.parametrize("kw", [dict(), dict(top_k=3), dict(top_p=0.7), dict(min_p=0.3)])
def test_verified_tokens_follow_the_target(kw):
    """One draft: the committed first token is distributed as the truncated target, whatever the
    drafter.  Exactly: over a grid of uniforms the acceptances and draws cover p."""
    rng = np.random.default_rng(5)
    V = 6
    q = tr.truncate(rng.normal(size=V), **kw)[4]
    p = np.stack([tr.truncate(rng.normal(size=V), **kw)[4] for _ in range(2)])
    got = np.zeros(V)
    N = 400
    grid = (np.arange(N) + 0.5) / N
    for x in np.flatnonzero(q > 0):
        hits = np.array([tr.accept([x], q[None], p, [u, 0.0])[0] for u in grid])
        got[x] += q[x] * hits.mean()
        miss = q[x] * (1 - hits.mean())
        if miss > 0:
            u0 = grid[hits == 0][0]
            nxt = [tr.accept([x], q[None], p, [u0, u])[1] for u in grid]
            got += miss * np.bincount(nxt, minlength=V) / N
    assert np.abs(got - p[0]).max() < 2 * V / N   # the grids' resolution
