"""The weights of 4-bit attention add up to one: where every key has the same
V, that V comes out bit for bit, whatever the scores."""
import numpy as np
import pytest
import torch

from kv_batches import Batch
from oracle import cache as ref
from paper_2609_34388_amd import binding

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")


def _equal_values(b, pool):
    """One V for all keys of a KV head, [Hkv, D]; written to every token that is read."""
    rng = np.random.default_rng(1)
    D = b.d
    row = ref.GRID[rng.integers(0, 8, (b.hkv, D))] * rng.choice([-1.0, 1.0], (b.hkv, D))
    row[:, ::32] = 6.0  # fixes the scales at one
    for r in range(b.R):
        page, slot = b.places(r, int(b.T[r]))
        for h in range(b.hkv):
            code, s = ref.encode(row[h])
            pool[page[:, None], h, ref._code_places(D, 1)[slot]] = code[0::2] + 16 * code[1::2]
            pool[page[:, None], h, ref._scale_places(D, 1)[slot]] = s
    return row


def _check(b, q, pool, row):
    """The products take the weights rounded to bf16, so the sum below them has
    to be of the rounded weights too: then both are fp32 sums of the same T < 6100
    weights, each off by at most T 2^-24 of itself (2^-11.4), and the quotient by
    less than 2^-10: less than the 2^-9 from a bf16 value to where it would round
    to a neighbour."""
    cache = torch.from_numpy(pool).to(DEV)
    br = b.branch_layout() if any(b.branches) else None
    out, _ = binding.kv4_attention(q.to(DEV), cache, b.layout4(cache), br)
    want = torch.from_numpy(np.repeat(row, b.g, axis=0)).to(torch.bfloat16).expand(b.rows, b.hq, b.d)
    bad = out.cpu() != want
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} elements"


BATCHES = {
    "blocks": [(5, 4, 8), (100, 3, 5), (0, 7, 9), (33, 0, 16), (257, 16, 0), (63, 1, 1)],
    "runs": [(6000, 2, 3), (900, 1, 0)],
    "branches": [(513, 8, [(2, 1, 9), (8, 0, 8)]), (100, 4, [(1, 1, 4), (3, 1, 6), (4, 0, 5)]), (300, 2, 3)],
    "prompt": [(40, 333, 0)],
}


@pytest.mark.parametrize("std", [1.0, 6.0])
@pytest.mark.parametrize("heads", [(8, 2, 128), (14, 2, 64)])
@pytest.mark.parametrize("name", list(BATCHES))
def test_equal_values_come_out_exactly(name, heads, std):
    b = Batch(BATCHES[name], heads=heads)
    q, pool = b.q(std), b.pool4()
    _check(b, q, pool, _equal_values(b, pool))


@pytest.mark.parametrize("heads", [(8, 2, 128), (14, 2, 64)])
def test_a_dominant_key_that_is_not_the_reference(heads):
    """Keys of score zero, then one of weight 2^10.5 to 2^12 against them: below
    where the running reference would move to it, so that its weight, nearly all
    of the row's, is rounded."""
    b = Batch([(150 + 5 * i, 1, 0) for i in range(24)], heads=heads)
    pool = b.pool4()
    D = b.d
    row = _equal_values(b, pool)
    # a key of ones scores D^-1/2 D mean(q)
    mean = np.linspace(7.35, 8.2, b.rows)[:, None, None] / np.sqrt(D)
    q = torch.from_numpy(mean + 0.01 * b.rng.standard_normal((b.rows, b.hq, D))).to(torch.bfloat16)
    one, s = ref.encode(np.ones(D))
    for r in range(b.R):
        page, slot = b.places(r, int(b.T[r]))
        for h in range(b.hkv):
            pool[page[:, None], h, ref._code_places(D, 0)[slot]] = 0
            pool[page[140], h, ref._code_places(D, 0)[slot[140]]] = one[0::2] + 16 * one[1::2]
            pool[page[140], h, ref._scale_places(D, 0)[slot[140]]] = s
    _check(b, q, pool, row)
