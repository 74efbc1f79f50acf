"""Attention mass of steps with more query columns than a work group holds at a
time, in batches long enough that it goes over them in turn."""
import numpy as np
import pytest
import torch

from kv_batches import PAGE, Batch
from paper_2609_34388_amd import binding
from test_gpu_evict import _check_mass, _lse, _pools16, _score_size, dev

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")

# Work groups of 256 keys that the batch gives a compute unit (256 of them): more
# than three of bf16 keys, more than eight of 4-bit ones.
BF16 = [(9000, 65, 3), (4000, 190, 0), (100, 5, 0), (701, 150, 2), (0, 64, 0), (0, 0, 0)]
KV4 = [(16400, 65, 3), (300, 100, 0), (50, 4, 0), (0, 128, 0), (31, 65, 1)]


@pytest.mark.parametrize("counted, decay", [(False, 1.0), (True, 0.75), (False, 0.0)])
@pytest.mark.parametrize("four, heads", [(False, (32, 16, 64)), (False, (32, 16, 128)), (True, (64, 32, 64)),
                                         (True, (64, 32, 128))])
def test_mass(four, heads, counted, decay):
    b = Batch(KV4 if four else BF16, heads=heads)
    q, lse = b.q(), _lse(b, b.rng)
    pool = b.pool4() if four else _pools16(b)
    count = b.rng.integers(-1, b.nv + 2) if counted else None
    if counted:
        count[0], count[1] = 64, 0  # 128 columns of 130; none
    old = b.rng.random((b.num_pages, b.hkv, PAGE)).astype(np.float32)
    if decay == 0.0:
        old[:] = np.nan
    mass, qd = dev(old), q.to(DEV)
    rc = None if count is None else torch.as_tensor(count, dtype=torch.int32, device=DEV)
    if four:
        cache = dev(pool)
        call = lambda m: binding.kv4_attention_mass(qd, cache, dev(lse), m, b.layout4(cache), row_count=rc, decay=decay)
    else:
        kd = pool[0].to(DEV)
        call = lambda m: binding.attention_mass(qd, kd, dev(lse), m, b.layout16(qd, kd), row_count=rc, decay=decay)
    again = mass.clone()
    call(mass), call(again)
    assert torch.equal(torch.nan_to_num(mass), torch.nan_to_num(again))  # a fixed order of sums
    want = b.mass(old, q, pool, lse, count, decay)
    touched = np.zeros(want.shape, dtype=bool)
    for r in range(b.R):
        page, slot = b.places(r, int(b.ctx[r] + b.nv[r]) if b.n[r] else 0)
        touched[page, :, slot] = True
    got = mass.cpu()
    assert np.array_equal(got.numpy()[~touched], old[~touched], equal_nan=True)
    _check_mass(torch.where(torch.from_numpy(touched), got, 0.0), np.where(touched, want, 0.0), old, b,
                None if count is None else np.clip(count, 0, b.nv), _score_size(b, q, pool))
