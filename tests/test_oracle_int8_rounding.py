"""What rounding to bf16 ahead of the 8-bit codes adds, from the two steps: up to a quarter to a half of a code's step within a
factor of two of a row's largest number, half as much for each factor of two below."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import int8 as oi


@pytest.mark.parametrize("top", [1.0, 1.0078125, 1.25, 1.5, 1.9921875])
@pytest.mark.parametrize("below", [0, 1, 2, 5])
def test_bf16_ahead_of_the_codes(top, below):
    a = np.float32(top)
    x = np.linspace(2.0 ** -below, min(top, 2.0) * 2.0 ** -below, 100001).astype(np.float32)
    step = float(a) / 127.0
    moved = np.abs(oi.bf16_round(x).astype(np.float64) - x).max() / step
    assert moved <= 127.0 / 256.0 / top * 2.0 ** -below * 1.0001
    if top > 1.0:      # (some number lies halfway between two bf16 ones)
        assert moved >= 0.24 * 2.0 ** -below


def test_codes_of_rounded_numbers():
    """Codes of a row and of the row rounded to bf16 first: at most one apart, and both within their distance of the number."""
    rng = np.random.default_rng(0)
    x = rng.normal(size=(200, 512)).astype(np.float32)
    q, s = oi.quantize_rows(x)
    b, sb = oi.quantize_rows(oi.bf16_round(x))
    assert np.abs(q.astype(int) - b).max() <= 1
    scale = np.abs(x).max(1, keepdims=True).astype(np.float64)
    off = np.abs(b * sb.astype(np.float64)[:, None] - x) / (scale / 127.0)
    assert 0.5 < off.max() <= 1.01
