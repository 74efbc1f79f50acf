"""Pins of the exact angles of far positions (no GPU)."""
from fractions import Fraction

import numpy as np

from oracle import window as ref

# Twice pi to 60 digits, and the Taylor series of sine and cosine in fractions.
TWO_PI = Fraction("6.28318530717958647692528676655900576839433879875021164194988918")


def exact_turn(position, freq):
    w = Fraction(int(position)) * Fraction(float(freq))
    w -= round(w / TWO_PI) * TWO_PI
    w = Fraction(round(w * 2 ** 80), 2 ** 80)
    c = s = Fraction(0)
    term, k = Fraction(1), 0
    while abs(term) > Fraction(1, 2 ** 80):
        if k % 2 == 0:
            c += term if k % 4 == 0 else -term
        else:
            s += term if k % 4 == 1 else -term
        k += 1
        term = Fraction(round(term * w / k * 2 ** 90), 2 ** 90)
    return c, s


def test_turns_of_far_positions():
    """Within 2^-62 for 80 bits' own rounding, at positions of 31 bits whose products
    need 55; the product in 64 bits is off by up to 2^-23 there."""
    rng = np.random.default_rng(4)
    position = np.concatenate([[0, 1, 2 ** 31 - 1, 2 ** 29 - 1], rng.integers(1 << 29, 1 << 31, 40)])
    freq = np.concatenate([[1.0], rng.uniform(0.3, 1.0, 7), 10000.0 ** -rng.uniform(0, 1, 4)]).astype(np.float32)
    c, s = ref.turns(position, freq)
    rounded = 0.0
    for i, p in enumerate(position):
        for j, f in enumerate(freq):
            wc, ws = exact_turn(p, f)
            for got, want in ((c[i, j], wc), (s[i, j], ws)):
                whole = np.float64(got)  # a long double as the sum of two doubles
                held = Fraction(float(whole)) + Fraction(float(got - np.longdouble(whole)))
                assert abs(held - want) <= Fraction(1, 2 ** 62)
            rounded = max(rounded, abs(float(Fraction(int(p)) * Fraction(float(f)) - Fraction(float(p) * float(f)))))
    assert 2.0 ** -24 < rounded <= 2.0 ** -23


def test_near_positions_need_no_more_than_64_bits():
    rng = np.random.default_rng(5)
    position = rng.integers(0, 1 << 29, 50)
    freq = (10000.0 ** (-np.arange(16) / 16)).astype(np.float32)
    x = rng.standard_normal((50, 2, 32))
    c, s = (t.astype(np.float64)[:, None] for t in ref.turns(position, freq))
    want = np.concatenate([x[..., :16] * c - x[..., 16:] * s, x[..., 16:] * c + x[..., :16] * s], -1)
    assert np.abs(ref.rotate(x, position, freq, False) - want).max() < 1e-14
