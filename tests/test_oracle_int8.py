"""Pins of the 8-bit integer and block-norm oracle: closed forms and properties that do not use its code."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import int8 as oi


def test_bf16_round_is_nearest_with_ties_to_even():
    for quarters, want in ((0, 0), (1, 0), (3, 1), (4, 1), (5, 1), (7, 2), (9, 2)):      # steps of 2^-7
        assert oi.bf16_round(np.float32(1 + quarters * 2.0 ** -9)) == 1 + want * 2.0 ** -7
    assert oi.bf16_round(np.float32(1 + 2.0 ** -8)) == 1.0 and oi.bf16_round(np.float32(1 + 3 * 2.0 ** -8)) == 1 + 2.0 ** -6
    assert np.isnan(oi.bf16_round(np.float32(np.nan))) and oi.bf16_round(np.float32(-np.inf)) == -np.inf


def test_codes_are_nearest_and_reach_127():
    rng = np.random.default_rng(0)
    x = rng.normal(size=(50, 128)).astype(np.float32) * np.exp(4 * rng.normal(size=(50, 1))).astype(np.float32)
    q, s = oi.quantize_rows(x)
    assert (np.abs(q).max(1) == 127).all()
    err = np.abs(x.astype(np.float64) - q * s.astype(np.float64)[:, None])
    assert (err <= (0.5 + 127 * 2.0 ** -22) * s.astype(np.float64)[:, None]).all()


def test_rows_of_zeros_tiny_and_not_finite():
    x = np.zeros((4, 128), np.float32)
    x[1, 3] = 2.0 ** -101
    x[2, 0], x[3, 5] = np.inf, np.nan
    q, s = oi.quantize_rows(x)
    assert s[0] == s[1] == np.float32(2.0 ** -100) / np.float32(127) and not q[0].any()
    assert q[1, 3] == 64 and np.count_nonzero(q) == 1 and np.isnan(s[2:]).all()      # 63.5 to even


def test_product_by_hand():
    x, w = np.array([[1, -2], [127, 127]], np.int8), np.array([[3, 4], [-127, -127]], np.int8)
    y = oi.product(x, np.array([0.5, 1], np.float32), w, np.array([2, 0.25], np.float32))
    np.testing.assert_array_equal(y, [[-5.0, 127 * 0.125], [889 * 2.0, -32258 * 0.25]])


@pytest.mark.parametrize("wide", [False, True])
def test_stream_and_next_input(wide):
    x = np.full((1, 4), 3.0, np.float32)
    y = np.array([[3.0, -3.0, 3.0, -3.0]], np.float32)
    u = oi.stream(x, y, np.ones(4, np.float32), np.full((1, 4), 2.0, np.float32), 0.5, 1e-30, wide)
    np.testing.assert_allclose(u, [[3.5, -0.5, 3.5, -0.5]], rtol=1e-6)      # 1.5 +- 2
    n = oi.next_input(u, np.full(4, 2.0, np.float32), 1e-30)
    np.testing.assert_allclose(n, 2 * u / 2.5, rtol=2.0 ** -8)               # root of 12.5 / 2
    np.testing.assert_array_equal(oi.stream(x, None, None, None, -1.0, 1.0, wide), -x)


def test_joined_by_hand():
    rows = np.arange(8, dtype=np.float32).reshape(4, 2)
    y, ay = oi.joined(rows, [0, 2, 2, 3], [3, 0, 1], np.array([0.5, 2.0, -1.0], np.float32), None)
    np.testing.assert_array_equal(y, [[3.0, 5.5], [0, 0], [-2.0, -3.0]])
    np.testing.assert_array_equal(ay, [[3.0, 5.5], [0, 0], [2.0, 3.0]])


def test_swiglu_is_near_the_real_expert():
    """Rounding to 8 bits four times moves a random expert by about a hundredth."""
    rng = np.random.default_rng(1)
    x, g, u, d = (rng.normal(size=s).astype(np.float32) * f for s, f in (((9, 256), 1), ((128, 256), .1), ((128, 256), .1),
                                                                         ((256, 128), .1)))
    y, tol = oi.swiglu_rows(*oi.quantize_rows(x), *(oi.quantize_rows(w) for w in (g, u, d)))
    a = x @ g.T
    ref = (a / (1 + np.exp(-a)) * (x @ u.T)) @ d.T
    assert 1e-3 < np.linalg.norm(y - ref) / np.linalg.norm(ref) < 3e-2
    assert np.isfinite(tol).all() and np.median(tol) < 1e-2 * np.abs(ref).max()
