"""The 4-bit cache on the GPU: rows in and out bit for bit, attention against
64 bits.  Slots that no request reads hold bytes of 0xff (scales of infinity)."""
import numpy as np
import pytest
import torch

from kv_batches import PAGE, Batch, check_attention
from oracle import cache as ref
from paper_2609_34388_amd import binding
from paper_2609_34388_amd import workloads as W

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")


def dev(x):
    return torch.from_numpy(x).to(DEV) if isinstance(x, np.ndarray) else x.to(DEV)


# ---------------------------------------------------------------------------
def _append_reference(b, pool, k, v):
    kx, vx = ref.bf16_values(W.bf16_bits(k)), ref.bf16_values(W.bf16_bits(v))
    for r in range(b.R):
        page, slot = b.places(r, int(b.n[r]), int(b.ctx[r]))
        for i in range(int(b.n[r])):
            row = int(b.q_indptr[r]) + i
            for h in range(b.hkv):
                ref.write_token(pool, page[i], h, slot[i], 0, kx[row, h])
                ref.write_token(pool, page[i], h, slot[i], 1, vx[row, h])
    return pool


@pytest.mark.parametrize("heads", [(4, 2, 128), (4, 4, 64), (3, 3, 128), (1, 1, 64)])
@pytest.mark.parametrize("requests", [[(0, 1, 0)], [(5, 2, 1), (0, 0, 0), (16, 1, 0), (31, 3, 14), (100, 0, 0), (7, 40, 0)]])
def test_append_and_read(heads, requests):
    b = Batch(requests, heads=heads)
    # parts of one projection: rows further apart than they are wide
    qkv = b.normal(b.rows, b.hq + 2 * b.hkv, b.d)
    qkv *= torch.exp2(torch.from_numpy(b.rng.integers(-12, 12, (1, 1, b.d)).astype(np.float32))).to(torch.bfloat16)
    k, v = qkv[:, b.hq:b.hq + b.hkv], qkv[:, b.hq + b.hkv:]
    pool = np.full((b.num_pages, b.hkv, 17 * b.d), 0xff, dtype=np.uint8)
    cache = dev(pool)
    on = qkv.to(DEV)
    lay = b.layout4(cache)
    binding.kv4_append(on[:, b.hq:b.hq + b.hkv], on[:, b.hq + b.hkv:], cache, lay)
    want = _append_reference(b, pool.copy(), k, v)
    assert (cache.cpu().numpy() == want).all()  # untouched bytes included
    kr, vr = binding.kv4_read(cache, lay)
    for got, x in ((kr, k), (vr, v)):
        code, s = ref.encode(ref.bf16_values(W.bf16_bits(x)))
        assert (got.double().cpu().numpy() == ref.decode(code, s)).all()


def test_append_every_finite_value():
    """Every finite bf16 value as the largest of a group and below a larger one."""
    bits = np.arange(1 << 16, dtype=np.uint32)
    x = torch.from_numpy(bits.astype(np.uint16).view(np.int16).copy()).view(torch.bfloat16)
    x = x[torch.isfinite(x.float())]
    rows = x.numel() // 64
    b = Batch([(0, rows, 0)], heads=(1, 1, 64))
    k = x[:rows * 64].reshape(rows, 1, 64)  # neighbours: one scale per group
    v = k.reshape(-1)[torch.from_numpy(b.rng.permutation(rows * 64))].reshape(rows, 1, 64)
    # mixed magnitudes within 2^8 of the group's largest
    v = torch.where(v.float().abs() > 0, v, torch.ones_like(v))
    cache = torch.full((b.num_pages, 1, 17 * 64), 0xff, dtype=torch.uint8, device=DEV)
    binding.kv4_append(k.to(DEV), v.to(DEV), cache, b.layout4(cache))
    kr, vr = binding.kv4_read(cache, b.layout4(cache))
    for got, want in ((kr, k), (vr, v)):
        code, s = ref.encode(ref.bf16_values(W.bf16_bits(want)))
        assert (got.double().cpu().numpy() == ref.decode(code, s)).all()


def test_append_twice_keeps_the_first_rows():
    b = Batch([(3, 6, 0), (30, 5, 0)], heads=(2, 2, 128))
    first, second = (b.normal(b.rows, 2, 128).to(DEV) for _ in range(2))
    cache = torch.zeros(b.num_pages, 2, 17 * 128, dtype=torch.uint8, device=DEV)
    lay = b.layout4(cache)
    binding.kv4_append(first, first, cache, lay)
    before, _ = binding.kv4_read(cache, lay)
    # one more row behind each request's
    c = Batch([(9, 1, 0), (35, 1, 0)], heads=(2, 2, 128))
    c.page_indptr, c.page_indices, c.num_pages = b.page_indptr, b.page_indices, b.num_pages
    binding.kv4_append(second[:2], second[:2], cache, c.layout4(cache))
    after, _ = binding.kv4_read(cache, lay)
    assert torch.equal(before, after)


# ---------------------------------------------------------------------------
def _attend(b, q, pool, **kw):
    cache = dev(pool)
    br = b.branch_layout() if any(b.branches) else None
    out, lse = binding.kv4_attention(q.to(DEV), cache, b.layout4(cache), br, **kw)
    torch.cuda.synchronize()
    return out, lse


def _score_size(b, q, pool):
    """Largest sum of |q_d k_d| scale over a row: at most |q| |k| scale."""
    size = 0.0
    for r in range(b.R):
        if b.n[r]:
            for h in range(b.hkv):
                size = max(size, np.linalg.norm(b.q_of(q, r, h), axis=-1).max() *
                           np.linalg.norm(b.keys_of(pool, r, h, int(b.T[r])), axis=-1).max())
    return size * b.d ** -0.5


BATCHES = {
    "one token": [(0, 1, 0)],
    "two keys": [(1, 1, 0)],
    "page end": [(15, 1, 0), (16, 1, 0), (31, 1, 0), (32, 1, 0), (127, 1, 0), (128, 1, 0)],
    "blocks": [(5, 4, 8), (100, 3, 5), (0, 7, 9), (33, 0, 16), (257, 16, 0), (0, 0, 0), (63, 1, 1)],
    "long": [(3000, 5, 11), (700, 16, 16)],
    "branches": [(100, 4, [(1, 1, 4), (3, 1, 6), (4, 0, 5)]), (7, 3, 0), (0, 2, [(0, 0, 3), (1, 0, 3), (2, 0, 3)]),
                 (513, 8, [(2, 1, 9), (8, 0, 8)]), (40, 0, [(0, 0, 6)]), (20, 5, 4)],
    "quadratic": [(300, 15, [(a, 0, 16) for a in range(16)])],
}


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 128), (9, 3, 128), (14, 2, 64), (4, 1, 64), (16, 1, 128)])
@pytest.mark.parametrize("name", list(BATCHES))
def test_attention(name, heads):
    b = Batch(BATCHES[name], heads=heads)
    q, pool = b.q(), b.pool4()
    out, lse = _attend(b, q, pool)
    check_attention(out, lse, *b.attention(q, pool), _score_size(b, q, pool))


@pytest.mark.parametrize("std", [0.0, 8.0])
def test_attention_flat_and_sharp(std):
    """All scores equal, and one key far above the rest."""
    b = Batch([(700, 3, 4), (90, 1, 0)])
    q, pool = b.q(std), b.pool4()
    out, lse = _attend(b, q, pool)
    check_attention(out, lse, *b.attention(q, pool), _score_size(b, q, pool))


def test_attention_of_many_requests():
    """More requests than a launch takes, in both forms, some of them empty."""
    rng = np.random.default_rng(5)
    plain = [(int(rng.integers(0, 90)), int(rng.integers(0, 3)), int(rng.integers(0, 4))) for _ in range(300)]
    b = Batch(plain, heads=(4, 2, 64))
    q, pool = b.q(), b.pool4()
    check_attention(*_attend(b, q, pool), *b.attention(q, pool), _score_size(b, q, pool))
    branched = [(c, 2, [(1, 1, 3), (2, 0, 2)] if i % 3 else 2) for i, (c, _, _) in enumerate(plain[:150])]
    b = Batch(branched, heads=(4, 2, 64))
    q, pool = b.q(), b.pool4()
    check_attention(*_attend(b, q, pool), *b.attention(q, pool), _score_size(b, q, pool))


def test_attention_split_over_many_runs():
    """One request's keys over many work groups, and a long one beside short ones."""
    for requests in ([(6000, 2, 3)], [(9000, 1, 0)] + [(40, 1, 0)] * 20):
        b = Batch(requests, heads=(4, 1, 128))
        q, pool = b.q(), b.pool4()
        need = binding.kv4_attention_workspace_bytes(b.layout4(dev(pool)))
        assert need > 0
        ws = torch.full((need,), 0xff, dtype=torch.uint8, device=DEV)  # needs no initialisation
        check_attention(*_attend(b, q, pool, workspace=ws), *b.attention(q, pool), _score_size(b, q, pool))


def test_attention_matches_the_bf16_cache():
    """The same values in a bf16 cache give the same attention within both
    kernels' bounds."""
    b = Batch([(500, 4, 8), (77, 2, 2)])
    q, pool = b.q(), b.pool4(poison=0)
    out, lse = _attend(b, q, pool)
    kv = [torch.zeros(b.num_pages, b.hkv, PAGE, b.d), torch.zeros(b.num_pages, b.hkv, b.d, PAGE)]
    for page in range(b.num_pages):
        for h in range(b.hkv):
            kv[0][page, h] = torch.from_numpy(ref.read_page(pool, page, h, 0))
            kv[1][page, h] = torch.from_numpy(ref.read_page(pool, page, h, 1)).T
    kc, vc = (x.to(torch.bfloat16).to(DEV) for x in kv)
    o16, l16 = binding.draft_verify_attention(q.to(DEV), kc, vc, b.q_indptr, b.nv, b.ctx, b.page_indptr,
                                              b.device_pages(DEV))
    _, _, mag = b.attention(q, pool)
    assert ((out.double() - o16.double()).abs().cpu().numpy() <= 4.1 * 2.0 ** -8 * mag + 1e-6).all()
    assert (lse - l16).abs().max() <= 2.0 ** -8  # that kernel's sum adds rounded weights


def test_attention_scale_and_outputs():
    b = Batch([(50, 2, 3)])
    q, pool = b.q(), b.pool4()
    cache = dev(pool)
    out = torch.empty(b.rows, b.hq, b.d, dtype=torch.bfloat16, device=DEV)
    got, lse = binding.kv4_attention(q.to(DEV), cache, b.layout4(cache, sm_scale=0.25), out=out, want_lse=False)
    assert got is out and lse is None
    check_attention(out, None, *b.attention(q, pool, scale=0.25), 1.0)


def test_attention_on_another_stream():
    b = Batch([(3000, 2, 2), (10, 1, 0)])
    q, pool = b.q(), b.pool4()
    cache, qd = dev(pool), q.to(DEV)
    lay = b.layout4(cache)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out, lse = binding.kv4_attention(qd, cache, lay, stream=s, workspace=torch.empty(
        binding.kv4_attention_workspace_bytes(lay), dtype=torch.uint8, device=DEV))
    s.synchronize()
    check_attention(out, lse, *b.attention(q, pool), _score_size(b, q, pool))


def test_empty_batches():
    b = Batch([(5, 0, 0), (0, 0, 0)])
    cache = torch.zeros(b.num_pages, b.hkv, 17 * b.d, dtype=torch.uint8, device=DEV)
    lay = b.layout4(cache)
    e = torch.empty(0, b.hq, b.d, dtype=torch.bfloat16, device=DEV)
    out, lse = binding.kv4_attention(e, cache, lay)
    assert out.shape == e.shape and lse.shape == (0, b.hq)
    binding.kv4_append(e[:, :b.hkv], e[:, :b.hkv], cache, lay)
    assert binding.kv4_read(cache, lay)[0].shape == (0, b.hkv, b.d)


def test_argument_checks():
    b = Batch([(5, 1, 0)])
    cache = torch.zeros(b.num_pages, b.hkv, 17 * b.d, dtype=torch.uint8, device=DEV)
    lay, q, k = b.layout4(cache), b.q().to(DEV), b.normal(b.rows, b.hkv, b.d).to(DEV)
    with pytest.raises(TypeError):
        binding.kv4_append(k.float(), k, cache, lay)
    with pytest.raises(ValueError):
        binding.kv4_append(k[:, :1], k, cache, lay)
    with pytest.raises(ValueError):
        binding.kv4_append(k, k, cache[:1], lay)
    with pytest.raises(ValueError):
        binding.kv4_append(torch.cat([k, k]), k, cache, lay)
    with pytest.raises(binding.RGError):  # rows that are no multiple of 16 bytes apart
        two = Batch([(5, 2, 0)])
        wide = torch.zeros(2, b.hkv * b.d + 4, dtype=torch.bfloat16, device=DEV)[:, :b.hkv * b.d].unflatten(1, (b.hkv, b.d))
        binding.kv4_append(wide, wide, torch.zeros(two.num_pages, b.hkv, 17 * b.d, dtype=torch.uint8, device=DEV),
                           two.layout4(torch.zeros(two.num_pages, b.hkv, 17 * b.d, dtype=torch.uint8, device=DEV)))
    with pytest.raises(TypeError):
        binding.kv4_attention(q.cpu(), cache, lay)
    with pytest.raises(ValueError):
        binding.kv4_attention(q[:, :4], cache, lay)
    with pytest.raises(ValueError):
        binding.kv4_attention(q, cache, lay, lse=torch.empty(1, dtype=torch.float32, device=DEV))
    with pytest.raises(binding.RGError):
        long = Batch([(9000, 1, 0)])
        pool = torch.zeros(long.num_pages, long.hkv, 17 * long.d, dtype=torch.uint8, device=DEV)
        binding.kv4_attention(q, pool, long.layout4(pool), workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError):
        binding.make_kv4_layout(8, cache[:, :, :100], b.q_indptr, b.nv, b.ctx, b.page_indptr, b.device_pages(DEV))


@pytest.mark.parametrize("heads", [(8, 1, 128), (16, 2, 64)])
def test_attention_of_many_columns_split(heads):
    """Full column groups and a last one, both cut into runs; with branches too."""
    for requests in ([(3000, 20, 14)], [(2000, 3, [(1, 0, 16), (2, 0, 16), (3, 0, 16)]), (17, 1, 0)]):
        b = Batch(requests, heads=heads)
        q, pool = b.q(), b.pool4()
        check_attention(*_attend(b, q, pool), *b.attention(q, pool), _score_size(b, q, pool))


def test_two_calls_at_once():
    """Two streams, a workspace each, the same cache."""
    b = Batch([(5000, 2, 2), (10, 1, 0)])
    q, pool = b.q(), b.pool4()
    cache, qd = dev(pool), q.to(DEV)
    lay = b.layout4(cache)
    need = binding.kv4_attention_workspace_bytes(lay)
    ws = [torch.empty(need, dtype=torch.uint8, device=DEV) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    torch.cuda.synchronize()
    for s, w in zip(streams, ws):
        got.append(binding.kv4_attention(qd, cache, lay, stream=s, workspace=w))
    torch.cuda.synchronize()
    want = b.attention(q, pool)
    for out, lse in got:
        check_attention(out, lse, *want, _score_size(b, q, pool))
    assert torch.equal(got[0][0], got[1][0])


def test_tensors_of_another_device(monkeypatch):
    """Kernels run on the current device: tensors elsewhere are refused."""
    b = Batch([(5, 1, 0)])
    cache = torch.zeros(b.num_pages, b.hkv, 17 * b.d, dtype=torch.uint8, device=DEV)
    lay, q, k = b.layout4(cache), b.q().to(DEV), b.normal(b.rows, b.hkv, b.d).to(DEV)
    slots = torch.zeros(b.num_pages, b.hkv, PAGE, device=DEV)
    el = binding.make_evict_layout(cache, [6], [3], b.page_indptr, b.device_pages(DEV))
    monkeypatch.setattr(binding, "_current_device", lambda: 1)
    for call in (lambda: binding.kv4_append(k, k, cache, lay), lambda: binding.kv4_read(cache, lay, k_out=k, v_out=k),
                 lambda: binding.kv4_attention(q, cache, lay),
                 lambda: binding.kv4_attention_mass(q, cache, torch.zeros(b.rows, b.hq, device=DEV), slots, lay),
                 lambda: binding.kv4_evict_tokens(cache, slots, slots.int(), el)):
        with pytest.raises(ValueError, match="current device"):
            call()


@pytest.mark.parametrize("heads, most", [((32, 8, 128), 6000), ((16, 16, 64), 9000), ((16, 16, 128), 6000)])
def test_attention_of_larger_batches(heads, most):
    """Larger batches of unlike requests: runs of every kind side by side."""
    rng = np.random.default_rng(11)
    plain = [(int(rng.integers(300, most)), int(rng.integers(1, 30)), int(rng.integers(0, 40))) for _ in range(9)]
    branched = [(c, 4, [(1, 1, 19), (3, 0, 19), (4, 0, 19)] if i % 2 else 3) for i, (c, _, _) in enumerate(plain)]
    for requests in (plain + [(5, 1, 0), (0, 0, 0), (0, 1, 0)], branched + [(0, 2, [(1, 0, 3)])]):
        b = Batch(requests, heads=heads)
        q, pool = b.q(), b.pool4()
        check_attention(*_attend(b, q, pool), *b.attention(q, pool), _score_size(b, q, pool))


@pytest.mark.parametrize("heads", [(6, 6, 64), (7, 7, 128)])
def test_append_and_read_of_many_blocks(heads):
    """So many that a work item takes several heads: as request by request,
    whose bytes test_append_and_read pins."""
    requests = [(5, 4000, 0), (16, 4096, 0), (0, 3333, 0), (31, 1, 0), (0, 0, 0), (100, 30, 0)]
    b = Batch(requests, heads=heads)
    k, v = (b.normal(b.rows, b.hkv, b.d).to(DEV) for _ in range(2))
    both = [torch.full((b.num_pages, b.hkv, 17 * b.d), 0xff, dtype=torch.uint8, device=DEV) for _ in range(2)]
    lay = b.layout4(both[0])
    binding.kv4_append(k, v, both[0], lay)
    pages = b.device_pages(DEV)
    rows = [slice(int(b.q_indptr[r]), int(b.q_indptr[r + 1])) for r in range(b.R)]
    one = []
    for r, (at, ctx) in enumerate(zip(rows, b.ctx)):
        n = at.stop - at.start
        half = n // 2  # two calls, the second behind the first
        for first, count in ((0, half), (half, n - half)):
            mine = torch.as_tensor(b.pages(r), device=DEV)
            l1 = binding.make_kv4_layout(b.hq, both[1], [0, count], [0], [int(ctx) + first], [0, len(mine)], mine)
            part = slice(at.start + first, at.start + first + count)
            binding.kv4_append(k[part], v[part], both[1], l1)
            one.append(binding.kv4_read(both[1], l1))
    assert torch.equal(both[0], both[1])
    kr, vr = binding.kv4_read(both[0], lay)
    assert torch.equal(kr, torch.cat([x for x, _ in one])) and torch.equal(vr, torch.cat([x for _, x in one]))


@pytest.mark.parametrize("heads", [(32, 1, 64), (5, 1, 128)])
def test_attention_of_other_groups(heads):
    b = Batch([(700, 2, 5), (31, 1, 0), (0, 9, 0)], heads=heads)
    q, pool = b.q(), b.pool4()
    check_attention(*_attend(b, q, pool), *b.attention(q, pool), _score_size(b, q, pool))


def test_append_and_read_of_many_requests():
    """More requests than a launch takes, some without rows."""
    b = Batch([(i % 37, i % 4, i % 3) for i in range(300)], heads=(2, 2, 64))
    k, v = (b.normal(b.rows, b.hkv, b.d) for _ in range(2))
    pool = np.full((b.num_pages, b.hkv, 17 * b.d), 0xff, dtype=np.uint8)
    cache = dev(pool)
    lay = b.layout4(cache)
    binding.kv4_append(k.to(DEV), v.to(DEV), cache, lay)
    assert (cache.cpu().numpy() == _append_reference(b, pool.copy(), k, v)).all()
    kr, _ = binding.kv4_read(cache, lay)
    code, s = ref.encode(ref.bf16_values(W.bf16_bits(k)))
    assert (kr.double().cpu().numpy() == ref.decode(code, s)).all()


@pytest.mark.parametrize("heads", [(8, 1, 64), (4, 2, 128)])
def test_attention_of_a_prompt(heads):
    """Many column groups: a prompt behind a short prefix, whole and in a batch."""
    for requests in ([(100, 700, 0)], [(0, 333, 0), (50, 3, 2), (17, 400, 16)]):
        b = Batch(requests, heads=heads)
        q, pool = b.q(), b.pool4()
        check_attention(*_attend(b, q, pool), *b.attention(q, pool), _score_size(b, q, pool))
