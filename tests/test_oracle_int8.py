"""Pins of the oracles of integer rows and of the 8-bit cache (CPU): brute force, closed forms, invariants."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import cache8, fp8, int8


def test_quantise_is_nearest_even_of_exact_quotients():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((40, 64)) * np.exp(rng.uniform(-60, 60, (40, 1)))).astype(np.float32)
    x[0] = np.float32(2.0 ** -149) * np.arange(64)
    x[1] = 0.0
    x[2, :4] = [127.0, 0.5, 1.5, -2.5]
    x[2, 4:] = 0.0
    q, s = int8.quantise(x)
    assert s[0] == s[1] == np.float32(2.0 ** -126) and not q[0].any() and not q[1].any()
    assert list(q[2, :4]) == [127, 0, 2, -2] and s[2] == 1.0
    for r in range(40):
        for c in range(64):
            f = Fraction(float(x[r, c])) / Fraction(float(s[r]))
            d = abs(f - int(q[r, c]))
            assert d < Fraction(1, 2) or (d == Fraction(1, 2) and q[r, c] % 2 == 0)


def test_quantise_marks_bad_rows():
    x = np.ones((3, 8), np.float32)
    x[1, 2], x[2, 7] = np.nan, -np.inf
    q, s = int8.quantise(x)
    assert np.isnan(s[1:]).all() and not q[1:].any() and (q[0] == 127).all()


def test_linear_is_the_scaled_sum():
    q, w = np.array([[1, -2], [127, 127]], np.int8), np.array([[3, 4]], np.int8)
    v = int8.linear(q, np.float32([0.5, 2]), w, np.float32([4]), np.float32([1]))
    assert v.tolist() == [[0.5 * 4 * -5 + 1], [2 * 4 * 889 + 1]]


def test_slots_are_a_permutation_that_keeps_fours_together():
    assert sorted(cache8.SLOTS) == list(range(64))
    assert all(cache8.slot(t + i) == cache8.slot(t) + i for t in range(0, 64, 4) for i in range(4))


def _empty(pages, heads, hd, table):
    z = lambda *s: np.full(s, 0x7F, np.uint8)  # noqa: E731
    return cache8.Cache(z(pages, heads, 64, hd), z(pages, heads, hd, 64), z(pages, heads), z(pages, heads), table)


def test_append_in_pieces_and_growth():
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((150, 64)), rng.standard_normal((150, 64))
    whole, parts = _empty(4, 2, 32, [[2, 0, 3]]), _empty(4, 2, 32, [[2, 0, 3]])
    whole.append(0, 0, k, v)
    for a, b in ((0, 1), (1, 60), (60, 130), (130, 150)):
        parts.append(0, a, k[a:b], v[a:b])
    assert np.array_equal(whole.ks[[2, 0, 3]], parts.ks[[2, 0, 3]])     # the scale of all a page's values, either way
    got, there = parts.rows(True, 0, 150, 1)
    assert there.all()
    step = 2.0 ** (parts.vs[[2, 0, 3], 1].astype(int) - 127)
    # half a step of each rounding: one where it came, one more if its page's scale grew
    assert np.all(np.abs(got - v[:, 32:]) <= 2 * np.maximum(2.0 ** -4 * np.abs(v[:, 32:]),
                                                              2.0 ** -10 * np.repeat(step, 64)[:150, None]))
    assert np.all(whole.k[1] == 0x7F) and np.all(whole.tile(False, 3, 0)[150 - 128:] == 0x7F)   # nothing else


def test_attention_of_known_answers():
    c = _empty(2, 1, 32, [[1, -1, 0]])
    k, v = np.zeros((130, 32)), np.zeros((130, 32))
    v[:64], v[128:] = 1.0, 4.0
    c.append(0, 0, k, v)
    out, mag, _ = c.attention(0, 130, np.ones((2, 64)), False)
    # the page in the middle is none: 64 tokens of 1 and two of 4 with equal weights
    assert np.allclose(out, (64 + 8) / 66) and np.allclose(mag, out)
    out, _, _ = c.attention(0, 130, np.ones((131, 64)), True)
    assert np.all(out[0] == 0.0) and np.allclose(out[1:65], 1.0) and np.allclose(out[130], 72 / 66)
    assert np.allclose(out[129], 68 / 65)


def test_codes_are_fp8s():
    assert cache8.fp8 is fp8
    with pytest.raises(AssertionError):
        fp8.encode(np.array([449.0]))
