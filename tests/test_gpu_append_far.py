"""Rotated appends at positions whose angles need more than 64 bits, on the GPU."""
import numpy as np
import pytest
import torch

from kv_batches import PAGE, Batch
from oracle import window as ref
from paper_2609_34388_amd import binding
from paper_2609_34388_amd import workloads as W

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_far_angles_are_exact(interleaved, kv8):
    """q and K of positions of 30 and 31 bits, bit for bit: cosine and sine of the
    exact angle in fp32, two products and a sum rounded to fp32, and to bf16 or to
    their block of 8 bits.  Elements whose cosine or sine lies within 1e-13 of a border
    of fp32, which the kernel's own 1e-14 may cross, are left out.  A product rounded to
    64 bits takes tens of q's elements to a neighbour."""
    rows, d, half = 2048, 64, 32
    b = Batch([(5, rows, 0)], heads=(6, 1, d))
    at = b.rng.integers(1 << 29, 1 << 31, rows)
    freq = (2.0 ** (-2.0 * np.arange(half) / d)).astype(np.float32)  # all above 2^-1
    x = b.normal(rows, 8, d)
    q, k, v = (t.to(DEV) for t in (x[:, :6], x[:, 6:7], x[:, 7:]))
    rot = binding.make_rotation(torch.from_numpy(freq).to(DEV), interleaved=interleaved,
                                positions=torch.as_tensor(at.astype(np.int32), device=DEV))
    pages = b.device_pages(DEV)
    if kv8:
        cache, scales = binding.new_kv8_cache(b.num_pages, 1, d, DEV)
        cache.zero_(), scales.fill_(2.0 ** -117)
        lay = binding.make_kv8_layout(6, cache, b.q_indptr, b.nv, b.ctx, b.page_indptr, pages)
        out = binding.kv8_append(k, v, cache, scales, lay, rotation=rot, q=q)
    else:
        kc = torch.zeros(b.num_pages, 1, PAGE, d, dtype=torch.bfloat16, device=DEV)
        vc = torch.zeros(b.num_pages, 1, d, PAGE, dtype=torch.bfloat16, device=DEV)
        lay = binding.make_layout(q, kc, b.q_indptr, b.nv, b.ctx, b.page_indptr, pages)
        out = binding.kv_append(k, v, kc, vc, lay, rotation=rot, q=q)
    got = out.cpu()
    if not kv8:
        page, slot = b.places(0, rows, 5)
        got = torch.cat([got, kc.cpu()[page, :, slot]], 1)
    c, s = ref.turns(at, freq)
    sure = np.ones((rows, 1, half), dtype=bool)
    for t in (c, s):
        sure &= ((t + 1e-13).astype(np.float32) == (t - 1e-13).astype(np.float32))[:, None]
    assert sure.mean() > 0.999
    c, s = (t.astype(np.float32)[:, None] for t in (c, s))
    y = x[:, :7].float().numpy()
    one, two = (y[..., 0::2], y[..., 1::2]) if interleaved else (y[..., :half], y[..., half:])
    first, second = one * c - two * s, two * c + one * s  # numpy rounds each step to fp32
    want = np.stack([first, second], -1).reshape(y.shape) if interleaved else np.concatenate([first, second], -1)
    sure = np.repeat(sure, 2, -1) if interleaved else np.concatenate([sure, sure], -1)
    other = W.bf16_bits(got) != W.bf16_bits(torch.from_numpy(want[:, :got.shape[1]]).to(torch.bfloat16))
    assert np.count_nonzero(other & sure) == 0
    if kv8:
        pool, ws = np.zeros(cache.shape, dtype=np.uint8), np.full(scales.shape, 2.0 ** -117)
        ref.append8(pool, ws, b.pages(0), 5, want[:, 6:].astype(np.float64), 0)
        assert (scales[..., 0].cpu().numpy() == ws[..., 0]).all()
        place = (*b.places(0, rows, 5), ref.place(d, 0))
        held, codes = (t[place[0][:, None], 0, place[2][place[1]]] for t in (cache.cpu().numpy(), pool))
        assert np.count_nonzero((held != codes) & sure[:, 0]) == 0
