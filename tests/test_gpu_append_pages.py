"""Appends of many pages at D = 128, on the GPU."""
import numpy as np
import pytest
import torch

from kv_batches import PAGE, Batch
from paper_2609_34388_amd import binding
from test_gpu_append import DEV, Rows, layout8, layout16, pools8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("heads", [(9, 3, 128), (10, 5, 128)])
def test_many_pages_of_long_rows(heads, kv8):
    """From 512 pages on, work groups of four of q's heads in the bf16 cache, else of
    eight; heads that are no multiple of either: the same bits as request by request."""
    b = Batch([(int(c), int(n), 0) for c, n in zip(range(0, 900, 5), [1, 7, 40, 0, 16, 170] * 30)], heads=heads)
    pages = (b.T + PAGE - 1) // PAGE - b.ctx // PAGE
    assert pages[b.n > 0].sum() >= 512
    x = Rows(b, 96, False)
    q, k, v = x.parts(x.qkv.to(DEV))
    if kv8:
        pool, s = pools8(b, poison=0)
        first = [torch.from_numpy(pool).to(DEV), torch.from_numpy(np.nan_to_num(s)).float().to(DEV)]
        call, lay = binding.kv8_append, layout8
    else:
        first = [b.normal(b.num_pages, b.hkv, PAGE, 128).to(DEV), b.normal(b.num_pages, b.hkv, 128, PAGE).to(DEV)]
        call, lay = binding.kv_append, layout16
    one = [t.clone() for t in first]
    out = call(k, v, *first, lay(b, first[0]), rotation=x.rotation(), q=q)
    for r in range(b.R):
        s = Batch([(int(b.ctx[r]), int(b.nv[r]), 0)], heads=heads)
        s.page_indptr = np.array([0, len(b.pages(r))], dtype=np.int32)
        s.page_indices, s.num_pages = b.pages(r), b.num_pages
        rows = slice(int(b.q_indptr[r]), int(b.q_indptr[r + 1]))
        got = call(k[rows], v[rows], *one, lay(s, one[0]), rotation=x.rotation(), q=q[rows])
        assert torch.equal(got, out[rows])
    assert all(torch.equal(a, c) for a, c in zip(first, one))
