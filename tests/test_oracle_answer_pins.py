"""Pins of the answering operators' reference: closed forms, invariants and brute force (CPU)."""
import math

import numpy as np
import pytest

from oracle import answer as A


def test_quantize_closed_forms():
    q, s = A.quantize_rows(np.array([[127.0, -127.0, 63.5, 64.5, 0.5, -0.5, 0.0]]), None, 1.0)
    np.testing.assert_array_equal(q, [[127, -127, 64, 64, 0, 0, 0]])      # halves to even
    assert s[0] == 1.0
    q, s = A.quantize_rows(np.zeros((1, 5)), np.ones(5), 1e-6)
    assert not q.any() and s[0] == 0
    q, s = A.quantize_rows(np.array([[1.0, np.nan], [np.inf, 1.0]]), None, 1.0)
    assert not q.any() and np.isnan(s).all()
    # RMSNorm: a row of one magnitude c is +-1 / sqrt(1 + eps / c^2) after the norm.
    q, s = A.quantize_rows(np.array([[3.0, -3.0, 3.0]]), np.ones(3), 0.25)
    np.testing.assert_array_equal(q, [[127, -127, 127]])
    assert s[0] == pytest.approx(1 / math.sqrt(1 + 0.25 / 9) / 127, rel=1e-15)


def test_quantize_is_scale_invariant_and_within_half_a_step():
    x = np.random.default_rng(0).standard_normal((4, 50))
    q, s = A.quantize_rows(x, None, 1.0)
    q2, s2 = A.quantize_rows(x * 1024.0, None, 1.0)
    np.testing.assert_array_equal(q, q2)
    np.testing.assert_array_equal(s * 1024.0, s2)
    assert np.all(np.abs(q * s[:, None] - x) <= 0.5000001 * s[:, None])


def test_linear_by_hand():
    a, w = np.array([[1, -2], [127, 3]], np.int8), np.array([[5, 6], [-128, 7], [0, 1]], np.int8)
    acc = [[sum(int(p) * int(q) for p, q in zip(r, c)) for c in w] for r in a]
    got = A.linear_i8(a, [2.0, 0.5], w, [1.0, 4.0, 0.25], [1.0, 0.0, -1.0])
    want = [[acc[i][j] * [2.0, 0.5][i] * [1.0, 4.0, 0.25][j] + [1.0, 0.0, -1.0][j] for j in range(3)] for i in range(2)]
    np.testing.assert_array_equal(got, np.array(want, np.float32))


def test_logprobs_closed_forms():
    o = A.logprobs(np.array([[2.0] * 8]), np.array([[0, 7, -1, 8]]), 3)
    np.testing.assert_allclose(o["token"][0, :2], -math.log(8), rtol=1e-15)
    assert o["token"][0, 2] == 0 and np.isnan(o["token"][0, 3])
    assert o["entropy"][0] == pytest.approx(math.log(8), rel=1e-15)
    np.testing.assert_array_equal(o["top_tokens"], [[0, 1, 2]])
    inf = np.inf
    o = A.logprobs(np.array([[-inf, 1.0, -inf], [-inf] * 3, [0.0, inf, 0.0]]), np.array([[1], [0], [0]]), 2)
    assert o["token"][0, 0] == 0 and o["token"][1, 0] == -inf and np.isnan(o["token"][2, 0])
    np.testing.assert_array_equal(o["top_tokens"], [[1, -1], [-1, -1], [-1, -1]])
    assert o["entropy"][0] == 0 and o["entropy"][1] == 0 and np.isnan(o["entropy"][2])


def test_logprobs_invariants():
    z = 3 * np.random.default_rng(1).standard_normal((3, 40))
    o = A.logprobs(z, np.tile(np.arange(40), (3, 1)), 40)
    np.testing.assert_allclose(np.exp(o["token"]).sum(1), 1, rtol=1e-14)
    np.testing.assert_allclose(-(np.exp(o["token"]) * o["token"]).sum(1), o["entropy"], rtol=1e-13)
    assert np.all(np.diff(o["top"], axis=1) <= 0)
    shifted = A.logprobs(z + 100.0, np.tile(np.arange(40), (3, 1)), 0)
    np.testing.assert_allclose(shifted["token"], o["token"], atol=1e-13)
