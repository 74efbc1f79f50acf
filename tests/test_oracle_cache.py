"""Hand-worked pins of the 64-bit forms behind the 4-bit cache, the attention
mass and the eviction (no GPU)."""
import numpy as np
import pytest

from oracle import cache as ref


def _group(*first):
    x = np.zeros(32)
    x[:len(first)] = first
    return x


def test_scale_follows_the_largest_magnitude():
    for top, b in ((4.0, 127), (6.9375, 127), (7.0, 128), (8.0, 128), (3.5, 127), (3.484375, 126), (1.0, 125), (0.0, 1),
                   (2.0 ** -126, 1), (1.99 * 2.0 ** 127, 252)):
        assert ref.encode(_group(top))[1].tolist() == [b], top


def test_codes_round_to_nearest_even():
    x = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5, -0.25, -0.75, -6.9375, 0.26, -0.0]
    code, b = ref.encode(_group(*x))
    assert b.tolist() == [127]
    assert code[:14].tolist() == [6, 0, 2, 2, 4, 4, 6, 6, 7, 8, 10, 15, 1, 8]
    assert ref.decode(code, b)[:8].tolist() == [4.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0]


@pytest.mark.parametrize("D", [64, 128])
def test_block_layout_uses_every_byte_once(D):
    places = np.concatenate([f(D, kv).ravel() for f in (ref._code_places, ref._scale_places) for kv in (0, 1)])
    assert sorted(places.tolist()) == list(range(17 * D))
    # spot values of the documented order
    assert ref._code_places(D, 0)[3, 33 % (D // 2)] == ((33 % (D // 2)) // 32) * 512 + 3 * 32 + (33 % (D // 2)) % 32
    assert ref._scale_places(D, 1)[9, 1] == 16 * D + D // 2 + (D // 32 + 1) * 8 + 1


def test_write_then_read():
    rng = np.random.default_rng(0)
    pool = np.full((2, 2, 17 * 64), 255, dtype=np.uint8)
    x = ref.GRID[rng.integers(0, 8, 64)] * rng.choice([-1.0, 1.0], 64)
    x[0], x[32] = 6.0, 4.0  # fixes both scales at 1
    ref.write_token(pool, 1, 0, 5, 1, x)
    assert (ref.read_page(pool, 1, 0, 1)[5] == x).all()
    assert (pool[0] == 255).all() and (pool[1, 1] == 255).all() and (pool[1, 0] != 255).sum() <= 34


def test_mass_of_equal_scores_is_the_share():
    q, K = np.zeros((2, 3, 64)), np.ones((6, 64))
    lse = np.stack([np.full(3, np.log(5.0)), np.full(3, np.log(6.0))])
    old = np.arange(6.0)
    got = ref.mass(old, q, K, lse, 4, 2, None, 0.5, 1.0)
    assert np.allclose(got, [0.5 * j + 3 / 5 + 3 / 6 for j in range(4)] + [3 / 5 + 3 / 6, 3 / 6])
    assert np.allclose(ref.mass(old, q, K, lse, 4, 2, 1, 0.0, 1.0), [3 / 5] * 5 + [0.0])


def test_evict_keeps_protected_then_best_then_lowest():
    score = np.array([9.0, 1.0, 1.0, 5.0, 1.0, 0.0, 7.0, 0.0])
    pos = np.arange(8)
    # position 7 is recent, 0 a sink; then 7.0, 5.0 and the first of the ones
    assert ref.evict(score, pos, 5, 1, 1, 8) == [(2, 6), (4, 7)]
    assert ref.evict(score, pos, 8, 1, 1, 8) == []
    assert ref.evict(score, pos, 0, 0, 0, 8) == []
    assert ref.evict(np.zeros(5), np.arange(5), 2, 0, 0, 5) == []


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_a_group_without_a_value_reads_as_nan(bad):
    x = np.concatenate([_group(1.0, bad, 2.0), _group(1.0, 4.0)])
    code, b = ref.encode(x)
    assert b.tolist() == [255, 127]
    got = ref.decode(code, b)
    assert np.isnan(got[:32]).all() and got[32:34].tolist() == [1.0, 4.0]
