"""Pins of the oracle for 8-bit products and token sampling (no GPU)."""
import numpy as np
import pytest

from oracle import eight_bit as eb
from oracle import tokens as tk

torch = pytest.importorskip("torch")


def test_e4m3_numbers_are_torchs():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(eb.e4m3_values(), codes)


def test_rounding_is_nearest_even():
    v = np.concatenate([np.random.default_rng(0).uniform(-448, 448, 4000),
                        np.random.default_rng(1).uniform(-0.05, 0.05, 4000),
                        [0.0, 2.0 ** -10, 3 * 2.0 ** -10, 448.0, 17.0, 19.0, 2.0 ** -6 * (1 + 1 / 16)]])
    v = v.astype(np.float32).astype(np.float64)
    want = torch.from_numpy(v).float().to(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(eb.e4m3_round(v), want)
    # and no number of the format is nearer than the one taken
    table = eb.e4m3_values()
    table = np.unique(table[np.isfinite(table)])
    far = np.abs(table[None] - v[:, None]).min(1)
    np.testing.assert_array_equal(np.abs(eb.e4m3_round(v) - v), far)


@pytest.mark.parametrize("amax, e", [(448.0, 0), (448.5, 1), (224.0, -1), (224.5, 0), (1.0, -8),
                                     (1.75, -8), (1.7500001, -7), (0.0, 0), (1e-40, -126)])
def test_scale_is_the_smallest_power_that_fits(amax, e):
    assert eb.scale_exponent(amax) == e


def test_quantised_block_is_within_half_a_step():
    x = np.random.default_rng(2).normal(size=(5, 256)) * np.exp(np.random.default_rng(3).normal(size=(5, 1)) * 5)
    q, e = eb.quantize_rows(x)
    s = np.repeat(2.0 ** e, 128, axis=1)
    assert (np.abs(q - x) <= np.maximum(np.abs(x) * 2.0 ** -4, 2.0 ** -10 * s)).all()
    assert (np.abs(q) <= 448 * s).all()


def test_sampling_frequencies_and_cuts():
    l = np.log([0.1, 0.4, 0.2, 0.3])
    got = [tk.sample_row(l, 1.0, 0, 1.0, 0.0, u)[0] for u in (0.0, 0.0999, 0.1001, 0.4999, 0.5001, 0.7001, 0.9999)]
    assert got == [0, 0, 1, 1, 2, 3, 3]
    assert list(tk.sample_row(l, 1.0, 2, 1.0, 0.0, 0.5)[2]) == [1, 3]
    assert list(tk.sample_row(l, 1.0, 0, 0.65, 0.0, 0.5)[2]) == [1, 3]
    assert list(tk.sample_row(l, 1.0, 0, 0.75, 0.0, 0.5)[2]) == [1, 2, 3]
    assert list(tk.sample_row(l, 1.0, 0, 1.0, 0.45, 0.5)[2]) == [1, 2, 3]
    assert list(tk.sample_row(l, 1.0, 3, 0.5, 0.0, 0.5)[2]) == [1, 3]      # 0.4 / 0.9 < 0.5
    token, conf, _, _ = tk.sample_row(l, 0.5, 0, 1.0, 0.0, 0.99)
    assert token == 3 and abs(conf - 0.3) < 1e-12                           # temperature 1
    assert tk.sample_row([1.0, 3.0, 3.0, 2.0], 0.0, 0, 1.0, 0.0, 0.9)[0] == 1
    assert list(tk.sample_row([0.0] * 6, 1.0, 0, 0.5, 0.0, 0.9)[2]) == [0, 1, 2]
    assert tk.sample_row([-np.inf, -np.inf], 1.0, 0, 1.0, 0.0, 0.5)[:2] == (-1, 0.0)
    assert tk.sample_row([0.0, np.inf, np.nan, np.inf], 1.0, 0, 1.0, 0.0, 0.5)[:2] == (3, 0.5)
