"""The oracles' bounds of an expert whose gates are far below zero: as narrow as elsewhere down to -87, and down to 0 below,
where SiLU may be taken as 0."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import eight_bit as eb
from oracle import int8 as oi


@pytest.mark.parametrize("eg", [0.0, 1e-6, 1e-3, 0.1, 0.9, 3.0])
def test_steepest_bounds_the_difference(eg):
    g = np.concatenate([np.linspace(-160, 40, 4001), [-700.0, 0.0, 700.0]])

    def silu(t):
        with np.errstate(over="ignore"):
            return t / (1.0 + np.exp(-t))
    with np.errstate(over="ignore"):
        bound = oi.steepest(g, np.full_like(g, eg), 1.0 / (1.0 + np.exp(-g))) * eg
    for t in np.linspace(-eg, eg, 41):
        diff = np.abs(silu(g + t) - silu(g))
        assert (diff <= bound * (1 + 1e-9) + 1e-12 * np.abs(silu(g))).all()      # (fp64's own roundings)


def expert(kind, gates):
    d = f = 128
    x, gate, up = np.zeros((2, d)), np.zeros((f, d)), np.zeros((f, d))
    x[:, 0], x[:, 1] = 1.0, [1.0, -2.0]
    gate[:, 0], up[:, 1] = np.where(np.arange(f) % 2, gates[0], gates[1]), 2.0 ** 60
    if kind == "e4m3":
        return eb.swiglu_rows(x, gate, up, np.eye(f))
    return oi.swiglu_rows(*oi.quantize_rows(x), *(oi.quantize_rows(w) for w in (gate, up, np.eye(f))))


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_results_of_low_gates_are_told_from_zero(kind):
    """Gates in the range: what was lost on the way does not pass."""
    y, tol = expert(kind, (-72.0, -80.0))
    large = np.abs(y) >= 0.99 * np.abs(y).max(1, keepdims=True)
    assert (y[large] != 0).all() and (tol[large] < 0.2 * np.abs(y)[large]).all()


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("gates", [(-104.0, -104.0), (-104.0, -88.0), (-96.0, -72.0)])
def test_zeros_below_the_range_are_allowed_and_move_their_own_results(kind, gates):
    y, tol = expert(kind, gates)
    below = np.tile(np.where(np.arange(128) % 2, gates[0], gates[1]) < -87.5, (2, 1))
    assert (tol[below] >= np.abs(y)[below]).all()
    assert (tol[~below] < 0.2 * np.abs(y)[~below]).all()


def test_silu_below_the_range():
    assert 87.0 * np.exp(-87.0) < 2.0 ** -119
