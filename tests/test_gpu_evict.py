"""Attention mass against 64 bits, eviction value for value, and the whole
round of calls as a serving loop makes them."""
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
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV) if isinstance(x, np.ndarray) else x.to(DEV)


def _pools16(b, std=1.0, poison=float("nan")):
    """bf16 K and V pools, `poison` in every slot no request reads."""
    k, v = b.normal(b.num_pages, b.hkv, PAGE, b.d, std=std), b.normal(b.num_pages, b.hkv, b.d, PAGE)
    live = torch.zeros(b.num_pages, PAGE, dtype=torch.bool)
    for r in range(b.R):
        page, slot = b.places(r, int(b.T[r]) if b.n[r] else 0)
        live[torch.from_numpy(page.astype(np.int64)), torch.from_numpy(slot)] = True
    k[~live[:, None, :, None].expand_as(k)] = poison
    v[~live[:, None, None, :].expand_as(v)] = poison
    return k, v


def _lse(b, rng):
    keys = np.concatenate([c + 1 + np.arange(n) for c, n in zip(b.ctx, b.n)]) if b.rows else np.zeros(0)
    return (np.log(keys)[:, None] + 0.5 + 0.1 * rng.standard_normal((b.rows, b.hq))).astype(np.float32)


def _check_mass(got, want, old, b, count, score_size=None):
    """A weight is exp of a difference of two numbers up to `size`: each is off
    by its fp32 sum (D 2^-24 of the terms' magnitude) and a few roundings, and
    n weights add up in fp32."""
    size = (b.d + 8) * 2.0 ** -24 * score_size + 2.0 ** -22 * (score_size + 16)
    rows = max(1, int((b.nv if count is None else count).max()) * b.g)
    tol = (size + (rows + 8) * 2.0 ** -24) * np.abs(want) + 1e-30
    bad = np.abs(got.double().cpu().numpy() - want) > tol
    assert not bad.any(), np.argwhere(bad)[:4]


def _score_size(b, q, pool):
    size = 1.0
    for r in range(b.R):
        V = int(b.nv[r])
        if V:
            for h in range(b.hkv):
                size = max(size, np.linalg.norm(b.q_of(q, r, h), axis=-1).max() *
                           np.linalg.norm(b.keys_of(pool, r, h, int(b.ctx[r]) + V), axis=-1).max() * b.d ** -0.5)
    return size


MASS = {
    "one token": [(0, 1, 0)],
    "tokens": [(15, 1, 0), (16, 1, 0), (255, 1, 0), (256, 1, 0), (300, 1, 2)],
    "blocks": [(5, 4, 8), (100, 3, 5), (0, 7, 9), (33, 0, 16), (257, 16, 0), (0, 0, 0), (63, 1, 1)],
    "prompt": [(0, 150, 0), (37, 77, 3), (600, 40, 0)],
    "branches": [(100, 4, [(1, 1, 4), (3, 1, 6), (4, 0, 5)]), (7, 3, 0)],
}


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64), (9, 3, 128), (14, 2, 64), (16, 1, 128)])
@pytest.mark.parametrize("name", list(MASS))
def test_mass(name, heads, four):
    b = Batch(MASS[name], heads=heads)
    q = b.q()
    pool = b.pool4() if four else _pools16(b)
    lse = _lse(b, b.rng)
    old = b.rng.random((b.num_pages, b.hkv, PAGE)).astype(np.float32)
    for count, decay in ((None, 1.0), (b.rng.integers(-1, b.nv + 2), 0.75), (None, 0.0)):
        start = old.copy()
        if decay == 0.0:
            start[:] = np.nan  # not read: nothing of it may stay where keys are
        mass = dev(start)
        rc = None if count is None else torch.as_tensor(count, dtype=torch.int32, device=DEV)
        if four:
            cache = dev(pool)
            binding.kv4_attention_mass(q.to(DEV), cache, dev(lse), mass, b.layout4(cache), row_count=rc, decay=decay)
        else:
            qd, kd = q.to(DEV), pool[0].to(DEV)
            binding.attention_mass(qd, kd, dev(lse), mass, b.layout16(qd, kd), row_count=rc, decay=decay)
        want = b.mass(start, q, pool, lse, count, decay)
        touched = np.zeros(want.shape, dtype=bool)
        for r in range(b.R):
            page, slot = b.places(r, int(b.ctx[r] + b.nv[r]) if b.n[r] else 0)
            touched[page, :, slot] = True
        got = mass.cpu()
        assert np.array_equal(got.numpy()[~touched], start[~touched], equal_nan=True)
        _check_mass(torch.where(torch.from_numpy(touched), got, 0.0), np.where(touched, want, 0.0), start, b,
                    None if count is None else np.clip(count, 0, b.nv), _score_size(b, q, pool))


def test_mass_of_many_requests():
    rng = np.random.default_rng(3)
    b = Batch([(int(rng.integers(0, 70)), int(rng.integers(0, 4)), int(rng.integers(0, 2))) for _ in range(200)],
              heads=(4, 2, 64))
    q, pool, lse = b.q(), _pools16(b), None
    lse = _lse(b, rng)
    count = rng.integers(0, b.nv + 1)
    old = rng.random((b.num_pages, b.hkv, PAGE)).astype(np.float32)
    qd, kd, mass = q.to(DEV), pool[0].to(DEV), dev(old)
    binding.attention_mass(qd, kd, dev(lse), mass, b.layout16(qd, kd), decay=0.5,
                           row_count=torch.as_tensor(count, dtype=torch.int32, device=DEV))
    want = b.mass(old, q, pool, lse, count, 0.5)
    _check_mass(mass, want, old, b, count, _score_size(b, q, pool))


def test_mass_sums_to_the_counted_rows():
    """With the attention's own lse the new weights of a head sum to rows x heads."""
    b = Batch([(900, 6, 0), (31, 2, 5)])
    q, pool = b.q(), b.pool4()
    cache, qd = dev(pool), q.to(DEV)
    lay = b.layout4(cache)
    _, lse = binding.kv4_attention(qd, cache, lay)
    first = torch.zeros(b.num_pages, b.hkv, PAGE, device=DEV)
    again = torch.zeros_like(first)
    binding.kv4_attention_mass(qd, cache, lse, first, lay)
    binding.kv4_attention_mass(qd, cache, lse, again, lay)
    assert torch.equal(first, again)  # a fixed order of sums
    for r in range(b.R):
        page, slot = b.places(r, int(b.ctx[r] + b.nv[r]))
        total = first.cpu().numpy()[page, :, slot].astype(np.float64).sum(axis=0)
        assert np.abs(total / (int(b.nv[r]) * b.g) - 1).max() < 1e-4


# ---------------------------------------------------------------------------
def _evict_reference(b, L, keep, tracked, evicted, sink, recent, score, arrays, positions):
    """Moves tokens of numpy pools: arrays as (pool, index of a token's data)."""
    pos_new = positions.copy()
    before = [a.copy() for a, _ in arrays]
    for r in range(b.R):
        n = int(L[r])
        page, slot = b.places(r, n)
        for h in range(b.hkv):
            pos = np.where(np.arange(n) < tracked[r], positions[page, h, slot], np.arange(n) + evicted[r])
            moves = ref.evict(score[page, h, slot], pos, int(keep[r]), sink, recent, n + int(evicted[r]))
            left = min(int(keep[r]), n)
            pos_new[page[:left], h, slot[:left]] = pos[:left]
            for to, src in moves:
                for (a, at), old in zip(arrays, before):
                    a[at(page[to], h, slot[to])] = old[at(page[src], h, slot[src])]
                pos_new[page[to], h, slot[to]] = pos[src]
    return pos_new


def _token_index(kind, D):
    if kind == "k":
        return lambda p, h, s: (p, h, s)
    if kind == "v":
        return lambda p, h, s: (p, h, slice(None), s)
    places = np.concatenate([f(D, kv) for f in (ref._code_places, ref._scale_places) for kv in (0, 1)], axis=1)
    return lambda p, h, s: (p, h, places[s])


def _evict_case(L, keep, heads, four, *, tracked=None, evicted=None, sink=0, recent=0, score=None, alias=False, mass=True,
                seed=0):
    b = Batch([(int(x), 0, 0) for x in L], heads=heads, seed=seed)
    rng = b.rng
    R = b.R
    tracked = np.zeros(R, int) if tracked is None else np.asarray(tracked)
    evicted = np.zeros(R, int) if evicted is None else np.asarray(evicted)
    shape = (b.num_pages, b.hkv, PAGE)
    if score is None:
        score = np.exp(2 * rng.standard_normal(shape)).astype(np.float32)
    else:
        score = score(rng, shape).astype(np.float32)
    m = score.copy() if alias else rng.random(shape).astype(np.float32)
    positions = np.full(shape, -7, dtype=np.int32)
    for r in range(R):  # a valid history: some positions below tracked + evicted, in any order
        t = int(tracked[r])
        page, slot = b.places(r, t)
        for h in range(b.hkv):
            positions[page, h, slot] = rng.permutation(t + int(evicted[r]))[:t]
    if four:
        pool = rng.integers(0, 256, (b.num_pages, b.hkv, 17 * b.d)).astype(np.uint8)
        arrays = [(pool.copy(), _token_index("4", b.d))]
    else:
        kv = [rng.integers(0, 1 << 16, s).astype(np.uint16) for s in
              ((b.num_pages, b.hkv, PAGE, b.d), (b.num_pages, b.hkv, b.d, PAGE))]
        arrays = [(kv[0].copy(), _token_index("k", b.d)), (kv[1].copy(), _token_index("v", b.d))]
    on = [torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).to(DEV) for a, _ in arrays]
    on = [t.view(torch.bfloat16) if t.dtype == torch.int16 else t for t in on]
    md, pd = dev(m), dev(positions)
    sd = md if alias else dev(score)
    lay = binding.make_evict_layout(on[0], L, keep, b.page_indptr, b.device_pages(DEV), tracked=tracked, evicted=evicted,
                                    sink=sink, recent=recent)
    kw = dict(mass=md) if mass else {}
    if four:
        binding.kv4_evict_tokens(on[0], sd, pd, lay, **kw)
    else:
        binding.evict_tokens(on[0], on[1], sd, pd, lay, **kw)
    torch.cuda.synchronize()
    if mass:
        arrays.append((m, lambda p, h, s: (p, h, s)))
        on.append(md)
    pos = _evict_reference(b, L, keep, tracked, evicted, sink, recent, score, arrays, positions)
    assert np.array_equal(pd.cpu().numpy(), pos)
    for (want, _), got in zip(arrays, on):
        if got.dtype == torch.bfloat16:
            assert np.array_equal(W.bf16_bits(got), want)
        else:
            assert np.array_equal(got.cpu().numpy(), want)
    if not mass:
        assert torch.equal(md.cpu(), torch.from_numpy(m))


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("heads", [(2, 2, 128), (3, 3, 64), (1, 1, 128)])
def test_evict(heads, four):
    L = [0, 1, 1, 2, 15, 16, 17, 64, 65, 100, 300, 1024, 1025]
    keep = [0, 0, 1, 1, 7, 16, 16, 1, 64, 99, 150, 1000, 40]
    _evict_case(L, keep, heads, four)
    _evict_case(L[7:], [20, 64, 99, 150, 1000, 40], heads, four, sink=4, recent=9)
    _evict_case(L[7:], [14, 14, 14, 14, 14, 14], heads, four, sink=5, recent=9)  # only the protected stay


@pytest.mark.parametrize("four", [False, True])
def test_evict_with_a_history(four):
    L, tracked, evicted = [200, 64, 500, 33], [150, 64, 0, 32], [1000, 5, 70, 0]
    _evict_case(L, [120, 40, 400, 33], (2, 2, 64), four, tracked=tracked, evicted=evicted, sink=8, recent=30)
    _evict_case(L, [120, 40, 400, 10], (2, 2, 128), four, tracked=tracked, evicted=evicted)


def _ties(rng, shape):
    return rng.integers(0, 3, shape)


def _signed(rng, shape):
    x = rng.standard_normal(shape)
    x[rng.random(shape) < 0.2] = 0.0
    x[rng.random(shape) < 0.2] = -0.0
    return x


def _extreme(rng, shape):
    return rng.choice(np.array([0.0, 1e-45, 1e-38, 3e38, -3e38, np.inf, -np.inf, 1.0, np.nextafter(np.float32(1), 2)]), shape)


@pytest.mark.parametrize("score", [_ties, _signed, _extreme, lambda rng, s: np.zeros(s)])
def test_evict_ties_and_signs(score):
    _evict_case([700, 90, 33], [400, 60, 32], (2, 2, 128), True, score=score, recent=7)
    _evict_case([700, 90, 33], [100, 1, 16], (2, 2, 64), False, score=score, sink=1)


def test_evict_scores_are_the_mass():
    _evict_case([700, 90], [400, 60], (2, 2, 128), True, alias=True, recent=7)
    _evict_case([700, 90], [400, 60], (2, 2, 128), False, mass=False)


def test_evict_many_and_long():
    rng = np.random.default_rng(1)
    L = rng.integers(0, 90, 230)
    _evict_case(L, np.minimum(L, rng.integers(4, 90, 230)), (2, 2, 64), True, sink=1, recent=3)
    _evict_case([40000], [25000], (1, 1, 64), True, sink=4, recent=100)


def test_evict_pads_its_calls():
    """Without its own arrays a call makes them; a workspace too small is refused."""
    b = Batch([(100, 0, 0)], heads=(2, 2, 64))
    cache = torch.zeros(b.num_pages, 2, 17 * 64, dtype=torch.uint8, device=DEV)
    pool = torch.zeros(b.num_pages, 2, PAGE, device=DEV)
    pos = torch.zeros(b.num_pages, 2, PAGE, dtype=torch.int32, device=DEV)
    lay = binding.make_evict_layout(cache, [100], [50], b.page_indptr, b.device_pages(DEV))
    with pytest.raises(binding.RGError):
        binding.kv4_evict_tokens(cache, pool, pos, lay, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(TypeError):
        binding.kv4_evict_tokens(cache, pool, pos.float(), lay)
    with pytest.raises(ValueError):
        binding.kv4_evict_tokens(cache, pool[:1], pos, lay)
    with pytest.raises(ValueError):
        binding.make_evict_layout(cache, [100], [50, 2], b.page_indptr, b.device_pages(DEV))
    with pytest.raises(ValueError):
        binding.make_evict_layout(pool[..., :5], [100], [50], b.page_indptr, b.device_pages(DEV))
    with pytest.raises(ValueError):
        binding.kv4_attention_mass(b.q().to(DEV), cache, torch.zeros(1, 2, device=DEV), pool, b.layout4(cache))


# ---------------------------------------------------------------------------
def _together(b, keep, sink, recent, steps):
    """A serving loop on both caches: rows in, attention, mass, eviction; every
    step's attention against 64 bits over the tokens that should be left."""
    R, hkv, d = b.R, b.hkv, b.d
    pages = b.device_pages(DEV)
    cache = torch.full((b.num_pages, hkv, 17 * d), 0xff, dtype=torch.uint8, device=DEV)
    mass = torch.full((b.num_pages, hkv, PAGE), float("nan"), device=DEV)
    pos = torch.zeros(b.num_pages, hkv, PAGE, dtype=torch.int32, device=DEV)
    L, tracked, evicted = (np.zeros(R, dtype=np.int64) for _ in range(3))
    # each (request, head)'s tokens by position: K, V, mass
    held = [[dict() for _ in range(hkv)] for _ in range(R)]
    order = [[[] for _ in range(hkv)] for _ in range(R)]  # position in each slot
    for rows in steps:
        n = np.asarray(rows)
        q_indptr = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        total = int(q_indptr[-1])
        q, k, v = b.normal(total, b.hq, d), b.normal(total, hkv, d), b.normal(total, hkv, d)
        lay = binding.make_kv4_layout(b.hq, cache, q_indptr, n, L, b.page_indptr, pages)
        qd = q.to(DEV)
        binding.kv4_append(k.to(DEV), v.to(DEV), cache, lay)
        out, lse = binding.kv4_attention(qd, cache, lay)
        binding.kv4_attention_mass(qd, cache, lse, mass, lay, decay=0.9)
        vals = []
        for x in (k, v):
            code, s = ref.encode(ref.bf16_values(W.bf16_bits(x)))
            vals.append(ref.decode(code, s))
        want, wlse, mag = (np.zeros(x.shape) for x in (out, lse, out))
        qx = ref.bf16_values(W.bf16_bits(q))
        for r in range(R):
            for h in range(hkv):
                for i in range(int(n[r])):
                    p = int(L[r] + evicted[r]) + i
                    held[r][h][p] = [vals[0][q_indptr[r] + i, h], vals[1][q_indptr[r] + i, h], 0.0]
                    order[r][h].append(p)
                if n[r] == 0:
                    continue
                K, V = (np.stack([held[r][h][p][c] for p in order[r][h]]) for c in (0, 1))
                at, heads = slice(int(q_indptr[r]), int(q_indptr[r + 1])), slice(h * b.g, (h + 1) * b.g)
                see = ref.visible(int(L[r]), int(n[r]), int(n[r]))
                want[at, heads], wlse[at, heads], mag[at, heads] = ref.attention(qx[at, heads], K, V, see, d ** -0.5)
                old = np.array([held[r][h][p][2] for p in order[r][h]])
                new = ref.mass(old, qx[at, heads], K, wlse[at, heads], int(L[r]), int(n[r]), None, 0.9, d ** -0.5)
                for p, w in zip(order[r][h], new):
                    held[r][h][p][2] = w
        check_attention(out, lse, want, wlse, mag, 4.0 * d ** 0.5)
        L = L + n
        got = mass.cpu().numpy()
        for r in range(R):
            page, slot = b.places(r, int(L[r]))
            for h in range(hkv):
                w = np.array([held[r][h][p][2] for p in order[r][h]])
                assert np.abs(got[page, h, slot] - w).max() <= 1e-4 * max(1.0, w.max())
        # cut by the GPU's own mass: equal sums would tie, so the reference uses its values
        el = binding.make_evict_layout(cache, L, keep, b.page_indptr, pages, tracked=tracked, evicted=evicted,
                                       sink=sink, recent=recent)
        binding.kv4_evict_tokens(cache, mass, pos, el, mass=mass)
        left = np.minimum(L, keep)
        where = pos.cpu().numpy()
        for r in range(R):
            page, slot = b.places(r, int(L[r]))
            for h in range(hkv):
                moves = ref.evict(got[page, h, slot], np.array(order[r][h]), int(keep[r]), sink, recent,
                                  int(L[r] + evicted[r]))
                o = order[r][h]
                for to, src in moves:
                    o[to] = o[src]
                del o[int(left[r]):]
                assert where[page[:len(o)], h, slot[:len(o)]].tolist() == o
        evicted, tracked, L = evicted + L - left, left.copy(), left
    return L


def test_a_serving_loop():
    b = Batch([(160, 0, 0), (96, 0, 0), (400, 0, 0)], heads=(8, 2, 128))
    left = _together(b, np.array([100, 64, 250]), 4, 20, [(120, 30, 300), (1, 1, 1), (8, 40, 5), (0, 16, 16), (1, 1, 1)])
    assert left.tolist() == [100, 64, 250]


def test_captured_round():
    """Append, attention, mass and eviction in a HIP graph: every replay as the
    eager calls, with eager work between replays."""
    b = Batch([(700, 3, 0), (65, 2, 0)], heads=(4, 2, 64), spare_pages_each=1)
    pool0 = dev(b.pool4(poison=0))
    q = b.q().to(DEV)
    k, v = (b.normal(b.rows, b.hkv, b.d).to(DEV) for _ in range(2))
    cache, mass = pool0.clone(), torch.zeros(b.num_pages, b.hkv, PAGE, device=DEV)
    pos = torch.zeros(b.num_pages, b.hkv, PAGE, dtype=torch.int32, device=DEV)
    lay = b.layout4(cache)
    el = binding.make_evict_layout(cache, b.T, [500, 60], b.page_indptr, b.device_pages(DEV), sink=2, recent=8)
    out, lse = torch.empty_like(q), torch.empty(b.rows, b.hq, device=DEV)
    ws = torch.empty(max(16, binding.kv4_attention_workspace_bytes(lay)), dtype=torch.uint8, device=DEV)
    ews = torch.empty(binding.evict_workspace_bytes(el), dtype=torch.uint8, device=DEV)

    def round_(stream=None):
        cache.copy_(pool0)
        mass.zero_()
        binding.kv4_append(k, v, cache, lay)
        binding.kv4_attention(q, cache, lay, out=out, lse=lse, workspace=ws)
        binding.kv4_attention_mass(q, cache, lse, mass, lay)
        binding.kv4_evict_tokens(cache, mass, pos, el, mass=mass, workspace=ews)

    round_()
    torch.cuda.synchronize()
    want = [x.clone() for x in (out, lse, mass, pos, cache)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        round_()
    for _ in range(3):
        for x in (out, lse):
            x.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip((out, lse, mass, pos, cache), want):
            assert torch.equal(got, w)
        q2 = q * 0.5
        binding.kv4_attention(q2, cache, lay, workspace=ws)
        torch.cuda.synchronize()


@pytest.mark.parametrize("four", [False, True])
def test_mass_of_keys_that_no_counted_row_sees(four):
    """Such keys add nothing, whatever they hold (here NaN, in 4 bits 2^128 and more)."""
    for heads, V in (((8, 2, 128), 8), ((16, 2, 64), 40)):  # few columns, and many
        b = Batch([(75, V, 3), (0, V, 0)], heads=heads)
        count = np.array([2, 0])
        q, lse = b.q(), _lse(b, b.rng)
        pool = b.pool4() if four else _pools16(b)
        places = ref._scale_places(b.d, 0) if four else None
        for r in range(b.R):
            page, slot = b.places(r, V - int(count[r]), int(b.ctx[r] + count[r]))
            for p, s in zip(page, slot):
                if four:
                    pool[p][:, places[s]] = 0xff
                else:
                    pool[0][int(p), :, s] = float("nan")
        mass = torch.full((b.num_pages, b.hkv, PAGE), 0.25, device=DEV)
        rc = torch.tensor(count, dtype=torch.int32, device=DEV)
        if four:
            cache = dev(pool)
            binding.kv4_attention_mass(q.to(DEV), cache, dev(lse), mass, b.layout4(cache), row_count=rc)
        else:
            qd, kd = q.to(DEV), pool[0].to(DEV)
            binding.attention_mass(qd, kd, dev(lse), mass, b.layout16(qd, kd), row_count=rc)
        got = mass.cpu().numpy()
        assert np.isfinite(got).all()
        for r in range(b.R):
            page, slot = b.places(r, V - int(count[r]), int(b.ctx[r] + count[r]))
            assert (got[page, :, slot] == 0).all()


def test_mass_of_long_runs():
    """Work items of several steps of 4-bit keys, the last of them incomplete."""
    b = Batch([(13009, 2, 0)], heads=(32, 32, 64))
    q, pool, lse = b.q(), b.pool4(), None
    lse = _lse(b, b.rng)
    old = b.rng.random((b.num_pages, b.hkv, PAGE)).astype(np.float32)
    cache, mass = dev(pool), dev(old)
    binding.kv4_attention_mass(q.to(DEV), cache, dev(lse), mass, b.layout4(cache), decay=0.5)
    want = b.mass(old, q, pool, lse, None, 0.5)
    page, slot = b.places(0, int(b.T[0]))
    _check_mass(mass.cpu()[page, :, slot], want[page, :, slot], old, b, None, _score_size(b, q, pool))


@pytest.mark.parametrize("L", [4096, 4097, 8192, 8193, 16384, 16385, 32769])
def test_evict_lengths(L):
    """Around the lengths at which a thread holds more slots."""
    _evict_case([L, 60], [L - 700, 54], (1, 1, 64), True, score=_ties, tracked=[L // 2, 0], evicted=[77, 0], sink=3, recent=50)
    _evict_case([L], [L // 3], (1, 1, 64), False, score=_signed, mass=False)


@pytest.mark.parametrize("four", [False, True])
def test_evict_one_page_partly_kept(four):
    """The page that holds slots on both sides of `keep`, token counts around it."""
    for L, keep in ((32, 17), (31, 23), (30, 24), (40, 25), (16, 9), (9, 8), (17, 15)):
        for heads in ((2, 2, 128), (2, 2, 64)):
            _evict_case([L, L], [keep, keep - 1], heads, four, seed=L)


@pytest.mark.parametrize("heads", [(32, 1, 64), (40, 2, 128), (10, 2, 64)])
def test_mass_of_other_groups(heads):
    """Query heads a KV head that do not divide 16 columns, or not 128."""
    for four in (False, True):
        b = Batch([(37, 77, 3), (0, 150, 0), (600, 2, 0)], heads=heads)
        q, lse = b.q(), _lse(b, b.rng)
        pool = b.pool4() if four else _pools16(b)
        old = b.rng.random((b.num_pages, b.hkv, PAGE)).astype(np.float32)
        mass, qd = dev(old), q.to(DEV)
        count = np.array([70, 150, 1])
        rc = torch.as_tensor(count, dtype=torch.int32, device=DEV)
        if four:
            cache = dev(pool)
            binding.kv4_attention_mass(qd, cache, dev(lse), mass, b.layout4(cache), row_count=rc)
        else:
            kd = pool[0].to(DEV)
            binding.attention_mass(qd, kd, dev(lse), mass, b.layout16(qd, kd), row_count=rc)
        want = b.mass(old, q, pool, lse, count, 1.0)
        for r in range(b.R):
            page, slot = b.places(r, int(b.ctx[r] + b.nv[r]))
            _check_mass(mass.cpu()[page, :, slot], want[page, :, slot], old, b, count, _score_size(b, q, pool))


def test_pools_past_32_bits():
    """The same pages at the far end of pools of more than 2^32 bytes."""
    hkv, d, far = 8, 128, 270000
    b = Batch([(300, 4, 3), (90, 2, 0), (517, 1, 0)], heads=(16, hkv, d), spare=0)
    n = b.num_pages
    q = b.q().to(DEV)
    k, v = (b.normal(b.rows, hkv, d).to(DEV) for _ in range(2))
    pool, (k16, v16) = dev(b.pool4()), (x.to(DEV) for x in _pools16(b, poison=0.0))
    lse, score = dev(_lse(b, b.rng)), dev(b.rng.random((n, hkv, PAGE)).astype(np.float32))
    keep = [200, 60, 400]

    def call(pages, cache, kc, vc, mass, mass16, pos, pos16):
        args = (b.q_indptr, b.nv, b.ctx, b.page_indptr, pages)
        lay, lay16 = binding.make_kv4_layout(16, cache, *args), binding.make_layout(q, kc, *args)
        binding.kv4_append(k, v, cache, lay)
        out = [*binding.kv4_read(cache, lay), *binding.kv4_attention(q, cache, lay)]
        binding.kv4_attention_mass(q, cache, lse, mass, lay)
        binding.attention_mass(q, kc, lse, mass16, lay16)
        out += [mass[-n:].clone(), mass16[-n:].clone()]
        for c, extra in ((cache, ()), (kc, (vc,))):
            el = binding.make_evict_layout(c, b.T, keep, b.page_indptr, pages, sink=2, recent=9)
            if extra:
                binding.evict_tokens(c, *extra, mass16, pos16, el, mass=mass16)
            else:
                binding.kv4_evict_tokens(c, mass, pos, el, mass=mass)
        return out + [x[-n:].clone() for x in (cache, kc, vc, mass, mass16, pos, pos16)]

    pages = b.device_pages(DEV)
    pos = torch.zeros(n, hkv, PAGE, dtype=torch.int32, device=DEV)
    near = [pool, k16, v16, score, score, pos, pos]
    want = call(pages, *(x.clone() for x in near))
    big = [torch.empty(far + n, *x.shape[1:], dtype=x.dtype, device=DEV) for x in near]
    for x, y in zip(big, near):
        x[far:] = y
    assert all(x.numel() * x.element_size() > 1 << 32 for x in big[:3])
    for got, w in zip(call(pages + far, *big), want):
        assert torch.equal(got.view(torch.int16) if got.dtype == torch.bfloat16 else got,
                           w.view(torch.int16) if w.dtype == torch.bfloat16 else w)


def test_own_tensors_on_another_stream():
    """Calls on a stream of their own that make their outputs and workspaces,
    while the current stream takes and fills memory."""
    b = Batch([(6000, 4, 3), (40, 1, 0)], heads=(8, 2, 128))
    q, pool0 = b.q().to(DEV), dev(b.pool4())
    L, keep = b.T, [4000, 20]

    def calls(stream):
        cache = pool0.clone()
        mass = torch.zeros(b.num_pages, b.hkv, PAGE, device=DEV)
        pos = torch.zeros(b.num_pages, b.hkv, PAGE, dtype=torch.int32, device=DEV)
        lay = b.layout4(cache)
        el = binding.make_evict_layout(cache, L, keep, b.page_indptr, b.device_pages(DEV), recent=8)
        if stream is not None:
            torch.cuda.synchronize()
        out, lse = binding.kv4_attention(q, cache, lay, stream=stream)
        noise = [torch.full((n,), 0x5a, dtype=torch.uint8, device=DEV) for n in (1 << 20, 1 << 22, 1 << 24, 1 << 25)]
        binding.kv4_attention_mass(q, cache, lse, mass, lay, stream=stream)
        del noise
        binding.kv4_evict_tokens(cache, mass, pos, el, mass=mass, stream=stream)
        noise = [torch.full((n,), 0x5a, dtype=torch.uint8, device=DEV) for n in (1 << 16, 1 << 18, 1 << 20, 1 << 22)]
        k, v = binding.kv4_read(cache, lay, stream=stream)
        torch.cuda.synchronize()
        return out, lse, mass, pos, cache, k, v

    want = calls(None)
    s = torch.cuda.Stream()
    for stream in (s, s.cuda_stream, s, s):
        for got, w in zip(calls(stream), want):
            assert torch.equal(got.view(torch.int16) if got.dtype == torch.bfloat16 else got,
                               w.view(torch.int16) if w.dtype == torch.bfloat16 else w)
