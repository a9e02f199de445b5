"""The distillation oracle against closed forms and central differences."""
import numpy as np
import pytest

from oracle import distill as od


def test_closed_forms():
    z = np.log(np.array([0.5, 0.25, 0.125, 0.125]))
    # one listed token, renormalised: p = 1, kl = -log q
    kl, g = od.slot_kl(z, [1], [7.0])
    np.testing.assert_allclose(kl, np.log(4))
    np.testing.assert_allclose(g, [0.5, -0.75, 0.125, 0.125])
    # with a bucket of the teacher's other half: p = (1/2, 1/2), q = (1/4, 3/4)
    kl, g = od.slot_kl(z, [1], [0.0], rest=0.0)
    np.testing.assert_allclose(kl, 0.5 * np.log(2) + 0.5 * np.log(2 / 3))
    np.testing.assert_allclose(g, [0.5 / 3, -0.25, 0.125 / 3, 0.125 / 3])
    np.testing.assert_allclose(g.sum(), 0, atol=1e-15)


def test_the_whole_vocabulary_listed_is_the_plain_divergence():
    rng = np.random.default_rng(0)
    z, t = rng.normal(size=9), rng.normal(size=9)
    kl, g = od.slot_kl(z, np.arange(9), t, T=2.0)
    p, q = od._softmax(t / 2), od._softmax(z / 2)
    np.testing.assert_allclose(kl, (p * np.log(p / q)).sum())
    np.testing.assert_allclose(g, (q - p) / 2, atol=1e-15)
    assert abs(od.slot_kl(t, np.arange(9), t)[0]) < 1e-15


def test_repeated_and_foreign_ids_are_no_entries():
    z = np.arange(5.0)
    a = od.slot_kl(z, [3, 1, 3, -1, 9], [1.0, 2.0, 50.0, 50.0, 50.0], rest=0.3)
    b = od.slot_kl(z, [3, 1], [1.0, 2.0], rest=0.3)
    assert a[0] == b[0] and np.array_equal(a[1], b[1])
    assert od.slot_kl(z, [-1, 7], [0.0, 0.0])[0] == 0
    assert od.slot_kl(z, [2], [-np.inf])[0] == 0


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("T", [1.0, 2.5])
def test_gradient_by_differences(rest, T):
    rng = np.random.default_rng(3)
    n, B, P, K, V = 2, 4, 2, 3, 11
    z = rng.normal(size=(n * B, V)) * 2
    ids = np.array([[rng.permutation(V)[:K] for _ in range(P)] for _ in range(n)])
    val = rng.normal(size=(n, P, K))
    r = rng.normal(size=(n, P)) if rest else None
    lab = rng.integers(0, V, (n, B - 1))
    lab[1, 1] = -100
    gl, gk, gc = [0.3, -0.7, 1.1], rng.normal(size=(n, P)), rng.normal(size=(n, B - 1))

    def f(z):
        kl, ce, loss, _ = od.distill(z, ids, val, r, lab, B, T, 0.5)
        return (np.array(gl) * loss).sum() + (gk * kl).sum() + (gc * ce).sum()

    grad = od.distill(z, ids, val, r, lab, B, T, 0.5, gl, gk, gc)[3]
    h = 1e-5
    for i in range(n * B):
        for v in range(V):
            e = np.zeros_like(z)
            e[i, v] = h
            np.testing.assert_allclose((f(z + e) - f(z - e)) / (2 * h), grad[i, v], atol=2e-9)
