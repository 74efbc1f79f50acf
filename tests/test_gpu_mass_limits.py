"""Attention mass of the most verify rows that a call takes: rows of q whose last
byte lies just below 2^31."""
import numpy as np
import pytest
import torch

from kv_batches import PAGE
from paper_2609_34388_amd import binding

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")


@pytest.mark.parametrize("four", [False, True])
def test_rows_up_to_the_bound(four):
    V, hq, hkv, D = 65535, 128, 8, 128
    g, pages = hq // hkv, (V + PAGE - 1) // PAGE
    gen = torch.Generator(device=DEV).manual_seed(5)
    q = torch.empty(V, hq, D, dtype=torch.bfloat16, device=DEV)
    assert 2 ** 31 - 2 ** 16 < q.numel() * 2 < 2 ** 31
    for i in range(0, V, 8192):
        q[i:i + 8192] = torch.randn(q[i:i + 8192].shape, generator=gen, device=DEV)
    keys = torch.randn(pages * PAGE, hkv, D, generator=gen, device=DEV).to(torch.bfloat16)
    lse = (torch.log(torch.arange(1, V + 1, device=DEV).float()) + 0.5)[:, None].expand(V, hq).contiguous()
    order = torch.from_numpy(np.random.default_rng(2).permutation(pages).astype(np.int32)).to(DEV)
    mass = torch.full((pages, hkv, PAGE), float("nan"), device=DEV)
    table = (np.array([0, V]), np.array([V]), np.array([0]), np.array([0, pages]), order)
    if four:
        cache = torch.zeros(pages, hkv, 17 * D, dtype=torch.uint8, device=DEV)
        lay = binding.make_kv4_layout(hq, cache, *table)
        binding.kv4_append(keys[:V], keys[:V], cache, lay)
        keys = binding.kv4_read(cache, lay)[0]  # as they are held
        binding.kv4_attention_mass(q, cache, lse, mass, lay, decay=0.0)
    else:
        pool = torch.empty(pages, hkv, PAGE, D, dtype=torch.bfloat16, device=DEV)
        pool[order.long()] = keys.reshape(pages, PAGE, hkv, D).transpose(1, 2)
        binding.attention_mass(q, pool, lse, mass, binding.make_layout(q, pool, *table), decay=0.0)
    # the first keys, some in the middle, and the last, which only the last rows see
    which = torch.tensor([0, 1, 31, 32, 63, 64, 40000] + list(range(V - 70, V)), device=DEV)
    for h in (0, hkv - 1):
        k = keys[which, h].double()
        want, size = torch.zeros(len(which), dtype=torch.float64, device=DEV), 0.0
        for i in range(0, V, 8192):
            x = q[i:i + 8192, h * g:(h + 1) * g].double()
            rows = torch.arange(i, min(i + 8192, V), device=DEV)
            w = torch.exp((x.reshape(-1, D) @ k.T.contiguous()).reshape(len(rows), g, -1) * D ** -0.5 -
                          lse[rows, h * g:(h + 1) * g, None].double())
            want += torch.where(rows[:, None, None] >= which, w, 0.0).sum((0, 1))
            size = max(size, float(x.norm(dim=-1).max() * k.norm(dim=-1).max()) * D ** -0.5)
        got = mass[order.long()[which // PAGE], h, which % PAGE].double()
        # a weight's exponent: D terms of total magnitude `size`, and the lse; then
        # a lane adds 16 weights of a tile, and the tiles of its wave, V g / 128
        tol = (D + 8) * 2.0 ** -24 * size + 2.0 ** -22 * (size + 16) + (V * g / 128 + 24) * 2.0 ** -24
        assert ((got - want).abs() <= tol * want).all(), float(((got - want).abs() / want).max())
