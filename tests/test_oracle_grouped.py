"""The oracle of the 8-bit activations and grouped weights against what defines it."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import grouped


def test_layout_is_the_documented_byte_of_every_value():
    rng = np.random.default_rng(0)
    for rows, K in ((1, 1), (3, 7), (2, 128), (5, 300)):
        codes = rng.integers(-127, 128, (rows, K), dtype=np.int8)
        flat = grouped.lay_out(codes)
        assert flat.size == -(-K // 128) * rows * 128
        seen = np.zeros(flat.size, bool)
        for r in range(rows):
            for k in range(K):
                at = ((k // 128) * rows + r) * 128 + (k % 128) // 8 * 8 + (k % 2) * 4 + (k % 8) // 2
                assert flat[at] == codes[r, k] and not seen[at]
                seen[at] = True
        assert not flat[~seen].any()


def test_codes_are_within_half_a_step_and_reach_the_grids_end():
    rng = np.random.default_rng(1)
    u = (rng.standard_normal((50, 333)) * np.exp(rng.normal(0, 20, (50, 1)))).astype(np.float32)
    codes, scale = grouped.quantize_rows(u)
    assert (np.abs(codes).max(1) == 127).all()
    # half a step, and two fp32 roundings of u * (127 / a), at most 127 in magnitude, and one of the scale: 127 * 3 * 2^-24 steps
    assert (np.abs(codes * scale.astype(np.float64)[:, None] - u) <= scale[:, None] * (0.5 + 127 * 4 * 2.0 ** -24)).all()


def test_rows_of_zeros_tiny_rows_and_rows_that_are_not_finite():
    u = np.zeros((6, 5), np.float32)
    u[1, 2], u[2, 0], u[3, 4], u[4] = np.inf, np.nan, -np.inf, np.float32(1e-38)
    u[5] = 2.0 ** -100
    codes, scale = grouped.quantize_rows(u)
    assert scale[0] == 0 and np.isnan(scale[1:4]).all() and not codes[:5].any()
    assert (codes[5] == 127).all() and scale[4] == scale[5] > 0


def test_silu_is_rounded_once():
    """Against exact rationals around the exponential's Taylor series."""
    for g in (-30.0, -3.140625, -0.5, 2.0 ** -20, 0.75, 1.0, 9.0, 88.0):
        x, term, e = Fraction(-g), Fraction(1), Fraction(1)
        for i in range(1, 400):
            term = term * x / i
            e += term
        want = Fraction(g) / (1 + e)
        got = Fraction(float(grouped.silu(np.float64(g))))
        assert abs(got - want) <= abs(want) * Fraction(1, 2 ** 24) * Fraction(1001, 1000)


@pytest.mark.parametrize("group", [32, 64, 128, 256, 1024])
def test_products_are_those_of_the_dequantized_matrices(group):
    rng = np.random.default_rng(group)
    codes, w = rng.integers(-127, 128, (4, 300), dtype=np.int8), rng.integers(-8, 8, (6, 300), dtype=np.int8)
    s, ws = rng.random(4).astype(np.float32), rng.random((-(-300 // group), 6)).astype(np.float32)
    y, mass = grouped.linear(codes, s, w, group, ws)
    full = w * np.repeat(ws.astype(np.float64), group, 0)[:300].T
    want = (codes * s.astype(np.float64)[:, None]) @ full.T
    assert np.allclose(y, want, rtol=1e-12, atol=1e-9) and (mass >= np.abs(y) * (1 - 1e-12)).all()
