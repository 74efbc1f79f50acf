"""Pins of the 64-bit references of rotated appends, the 8-bit cache and window
masks (no GPU)."""
import math

import numpy as np
import pytest
import torch

from oracle import cache, window as ref


def test_grid_is_e4m3():
    x = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(x, ref.GRID, equal_nan=True)


def test_codes_round_to_nearest_even():
    rng = np.random.default_rng(0)
    y = rng.standard_normal(20000) * np.exp(3 * rng.standard_normal(20000))
    mid = (ref.GRID[:126] + ref.GRID[1:127]) / 2  # ties
    y = np.clip(np.concatenate([y, mid, -mid, ref.GRID[:127], [0.0, -0.0, 448.0]]), -448, 448)
    y32 = y.astype(np.float32)
    want = torch.from_numpy(y32).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert (ref.codes(y32.astype(np.float64), 1.0) == want).all()
    assert (ref.codes(np.array([math.inf, -math.inf, math.nan]), 2.0) == 127).all()
    assert (ref.codes(np.array([1000.0, -1000.0]), 1.0) == [126, 254]).all()


def test_exponent_keeps_the_largest_within_448():
    for top in [1.0, 1.5, 1.749, 1.75, 1.99, 3.4e38, 1e-30, 2.0 ** -133, 0.0]:
        e = ref.exponent(top)
        assert -117 <= e <= 119
        if -117 < e < 119:
            assert 224 <= top / 2.0 ** e < 448


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_complex_product(interleaved):
    rng = np.random.default_rng(1)
    x, pos = rng.standard_normal((5, 3, 64)), np.array([0, 1, 7, 100000, 2 ** 31 - 1])
    freq = 10000.0 ** (-np.arange(16) / 16)
    y = ref.rotate(x, pos, freq, interleaved)
    assert (y[0] == x[0]).all() and (y[..., 32:] == x[..., 32:]).all()
    pairs = (lambda z: z[..., 0:32:2] + 1j * z[..., 1:32:2]) if interleaved else (lambda z: z[..., :16] + 1j * z[..., 16:32])
    want = pairs(x) * np.exp(1j * pos[:, None, None] * freq)
    assert np.abs(pairs(y) - want).max() < 1e-12
    # scores depend on the distance alone
    a, b = ref.rotate(x[:1], np.array([40]), freq, interleaved), ref.rotate(x[1:2], np.array([33]), freq, interleaved)
    c, d = ref.rotate(x[:1], np.array([7]), freq, interleaved), x[1:2]
    assert np.abs((a * b).sum(-1) - (c * d).sum(-1)).max() < 1e-11


def test_append_rounds_kept_tokens_at_a_larger_scale():
    pool, scales = np.zeros((2, 1, 32 * 64), dtype=np.uint8), np.zeros((2, 1, 2))
    rng = np.random.default_rng(2)
    first, second = rng.standard_normal((10, 1, 64)), 40 * rng.standard_normal((12, 1, 64))
    pages = np.array([1, 0])
    ref.append8(pool, scales, pages, 0, first, 0)
    held = ref.values(pool, scales, 1, 0, 0)[:10]
    assert np.abs(held - first[:, 0]).max() <= 2.0 ** -4 * np.abs(first).max()
    ref.append8(pool, scales, pages, 10, second, 0)
    assert scales[1, 0, 0] == 2.0 ** ref.exponent(np.abs(second[:6]).max()) and scales[1, 0, 1] == 0
    again = ref.values(pool, scales, 1, 0, 0)
    big = np.abs(held) >= 2.0 ** -6 * scales[1, 0, 0]
    assert (again[:10][big] == held[big]).all()
    assert np.abs(again[:10] - held).max() <= 2.0 ** -10 * scales[1, 0, 0]
    # a smaller row leaves scale and codes
    before = pool.copy()
    ref.append8(pool, scales, pages, 15, 0.01 * first[:1], 0)
    assert scales[1, 0, 0] == 2.0 ** ref.exponent(np.abs(second[:6]).max())
    at = ref.place(64, 0)
    assert (pool[1, 0][at[:15]] == before[1, 0][at[:15]]).all()


def test_places_cover_a_block():
    for D in (64, 128):
        both = np.concatenate([ref.place(D, 0).ravel(), ref.place(D, 1).ravel()])
        assert (np.sort(both) == np.arange(32 * D)).all()


def test_windows():
    no = ref.visible(5, 2, 6, [(1, 1, 2), (2, 0, 2)])
    assert (no == cache.visible(5, 2, 6, [(1, 1, 2), (2, 0, 2)])).all()
    assert (ref.visible(5, 2, 6, None, 100, 0) == cache.visible(5, 2, 6)).all()
    see = ref.visible(5, 2, 4, None, 3, 1)
    # row 0 (position 5): sink 0, positions 3, 4, 5; row 1: 4, 5, 6; draft rows (7, 8): 5, 6 and 6, and their block
    want = [[0, 3, 4, 5], [0, 4, 5, 6], [0, 5, 6, 7, 8], [0, 6, 7, 8]]
    assert [list(np.flatnonzero(r)) for r in see] == want
    # a branch that keeps one verify row (positions 6, 7), lead row first, window of one: its own rows only
    see = ref.visible(5, 2, 4, [(1, 1, 2)], 1, 0)[2:]
    assert [list(np.flatnonzero(r)) for r in see] == [[7], [7, 8]]
