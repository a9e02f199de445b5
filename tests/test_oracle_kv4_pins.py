"""Pins of the 4-bit cache's oracle: codes and scales by hand and by brute force, attention by
closed forms."""
import numpy as np
import pytest

from oracle import kv4


def test_codes_by_hand():
    y = [0.0, 0.2, 0.25, 0.26, 0.74, 0.75, 0.76, 1.25, 1.26, 1.75, 2.5, 2.51, 3.5, 3.49, 5.0, 5.01, 6, 9]
    want = [0, 0, 0, 1, 1, 2, 2, 2, 3, 4, 4, 5, 6, 5, 6, 7, 7, 7]
    assert kv4.codes(np.array(y)).tolist() == want
    assert kv4.codes(-np.array(y)).tolist() == want


@pytest.mark.parametrize("amax,e", [(7.0, 0), (7.0001, 1), (3.5, -1), (3.6, 0), (6.0, 0), (8.0, 1),
                                    (0.0, -125), (2.0 ** -140, -125), (3.38e38, 125)])
def test_key_exponents(amax, e):
    assert kv4.key_exponent(amax) == e


def test_value_scales():
    assert kv4.value_scale(6.0) == 1.0
    assert kv4.value_scale(6.01) == 1.0078125          # the next bfloat16 above 1
    assert kv4.value_scale(0.0) == 2.0 ** -126
    rng = np.random.default_rng(0)
    for a in np.abs(rng.standard_normal(200)) * 2.0 ** rng.integers(-90, 90, 200):
        s = kv4.value_scale(a)
        m, e = np.frexp(s)
        assert m * 256 == int(m * 256)                 # eight significant bits
        assert 6 * s >= a > 6 * (s - 2.0 ** (e - 8))   # and none smaller


def test_an_element_is_the_nearest_of_all_levels():
    rng = np.random.default_rng(1)
    v = rng.standard_normal((5, 64)) * 3
    got = kv4.quantise_values(v)
    k = kv4.quantise_keys(v)
    for i in range(5):
        s = kv4.value_scale(np.abs(v[i]).max())
        grid = np.concatenate([kv4.LEVELS, -kv4.LEVELS])
        assert np.array_equal(np.abs(v[i] - got[i]), np.abs(v[i][:, None] - grid * s).min(1))
        for b in (0, 32):
            u = 2.0 ** kv4.key_exponent(np.abs(v[i, b:b + 32]).max())
            assert np.array_equal(np.abs(v[i, b:b + 32] - k[i, b:b + 32]),
                                  np.abs(v[i, b:b + 32, None] - grid * u).min(1))


def test_what_is_no_number_spoils_its_scale_alone():
    v = np.ones((2, 64))
    v[1, 40] = np.inf
    k = kv4.quantise_keys(v)
    assert np.isfinite(k[0]).all() and np.isfinite(k[1, :32]).all() and np.isnan(k[1, 32:]).all()
    q = kv4.quantise_values(v)
    assert np.isfinite(q[0]).all() and np.isnan(q[1]).all()


def test_attention_of_equal_keys_is_the_mean():
    rng = np.random.default_rng(2)
    q = rng.standard_normal((2, 4, 8))
    k = np.ones((6, 2, 8))
    v = rng.standard_normal((6, 2, 8))
    out, lse, _, _ = kv4.attend(q, k, v)
    for h in range(4):
        assert np.allclose(out[:, h], v[:, h // 2].mean(0))
    assert np.allclose(lse, q.sum(2) / np.sqrt(8) + np.log(6))


def test_causal_slots_and_empty_rows():
    rng = np.random.default_rng(3)
    q, kb, vb = (rng.standard_normal((3, 1, 4)) for _ in range(3))
    none = np.zeros((0, 1, 4))
    out, lse, _, _ = kv4.attend(q, none, none, kb, vb, causal=True)
    assert np.allclose(out[0, 0], vb[0, 0])
    assert np.allclose(lse[0, 0], q[0, 0] @ kb[0, 0] / 2)
    out, lse, _, _ = kv4.attend(q, none, none)
    assert not out.any() and np.isneginf(lse).all()
