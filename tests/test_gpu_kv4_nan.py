"""Infinities and NaN in the rows of a 4-bit cache: their group of 32 elements
reads as NaN, and so do the rows of attention that see it."""
import numpy as np
import pytest
import torch

from kv_batches import PAGE, Batch
from oracle import cache as ref
from paper_2609_34388_amd import binding
from paper_2609_34388_amd import workloads as W

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
BITS = [0x7f80, 0xff80, 0x7f81, 0x7fff, 0xffff, 0xffc0]  # infinities, the smallest NaN, the largest, ...


@pytest.mark.parametrize("heads", [(4, 2, 128), (3, 3, 64)])
def test_append_marks_the_group(heads):
    b = Batch([(5, 40, 0), (0, 7, 0)], heads=heads)
    both = [b.normal(b.rows, b.hkv, b.d) for _ in range(2)]
    for x in both:
        for bits in BITS:
            at = tuple(b.rng.integers(0, (b.rows, b.hkv, b.d)))
            x.view(torch.int16)[at] = int(np.uint16(bits).astype(np.int16))
        x[3, 0, 1], x[3, 0, 2] = 3.38e38, -3.38e38  # finite: as before
    cache = torch.full((b.num_pages, b.hkv, 17 * b.d), 0xff, dtype=torch.uint8, device=DEV)
    lay = b.layout4(cache)
    binding.kv4_append(*(x.to(DEV) for x in both), cache, lay)
    for x, got in zip(both, binding.kv4_read(cache, lay)):
        code, s = ref.encode(ref.bf16_values(W.bf16_bits(x)))
        assert 1 <= (s == 255).sum() <= len(BITS)
        assert np.array_equal(got.double().cpu().numpy(), ref.decode(code, s), equal_nan=True)
    # the scale bytes themselves, where an eviction would move them
    pool = cache.cpu().numpy()
    for kv, x in enumerate(both):
        _, s = ref.encode(ref.bf16_values(W.bf16_bits(x)))
        for r in range(b.R):
            page, slot = b.places(r, int(b.n[r]), int(b.ctx[r]))
            for h in range(b.hkv):
                got = pool[page[:, None], h, ref._scale_places(b.d, kv)[slot]]
                assert np.array_equal(got, s[b.q_indptr[r]:b.q_indptr[r + 1], h])


@pytest.mark.parametrize("kv", [0, 1])
@pytest.mark.parametrize("heads", [(8, 2, 128), (14, 2, 64)])
@pytest.mark.parametrize("code", [0x00, 0x77, 0xf8])
def test_attention_and_mass_of_such_a_token(heads, kv, code):
    """A cached token of one request and KV head: every row of that head is NaN
    (where the token's V is, in that group of dims), no other is; its mass too."""
    b = Batch([(300, 3, 4), (90, 1, 0)], heads=heads)
    pool, q = b.pool4(), b.q()
    page, slot = b.places(0, 300)
    at = 217
    pool[page[at], 1, ref._code_places(b.d, kv)[slot[at]]] = code
    pool[page[at], 1, ref._scale_places(b.d, kv)[slot[at], 1]] = 255  # dims 32 .. 63
    cache = torch.from_numpy(pool).to(DEV)
    lay = b.layout4(cache)
    out, lse = binding.kv4_attention(q.to(DEV), cache, lay)
    want = np.zeros(out.shape, dtype=bool)
    want[:b.n[0], b.g:2 * b.g, slice(32, 64) if kv else slice(None)] = True
    assert np.array_equal(out.isnan().cpu().numpy(), want)
    assert torch.isfinite(out[~torch.from_numpy(want).to(DEV)]).all()
    hurt = np.zeros(lse.shape, dtype=bool)
    if kv == 0:
        hurt[:b.n[0], b.g:2 * b.g] = True
    assert np.array_equal(lse.isnan().cpu().numpy(), hurt)
    mass = torch.zeros(b.num_pages, b.hkv, PAGE, device=DEV)
    binding.kv4_attention_mass(q.to(DEV), cache, torch.full_like(lse, 6.0), mass, lay)
    got = mass.cpu().numpy()
    assert np.isnan(got).sum() == (1 - kv) and (kv == 1 or np.isnan(got[page[at], 1, slot[at]]))
