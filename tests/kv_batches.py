"""Ragged batches over paged caches for the tests of the 4-bit cache, the
attention mass and the eviction: host structure and seeded tensors."""
import numpy as np
import torch

from oracle import cache as ref
from paper_2609_34388_amd import binding
from paper_2609_34388_amd import workloads as W

PAGE = 16


class Batch:
    """Requests of (context, verify rows, draft rows or list of branches)."""

    def __init__(self, requests, heads=(8, 2, 128), seed=0, spare=3, spare_pages_each=0):
        self.hq, self.hkv, self.d = heads
        self.g = self.hq // self.hkv
        rng = np.random.default_rng([seed, len(requests), *heads])
        self.ctx = np.array([r[0] for r in requests], dtype=np.int32)
        self.nv = np.array([r[1] for r in requests], dtype=np.int32)
        self.branches = [list(r[2]) if isinstance(r[2], (list, tuple)) else None for r in requests]
        nd = [sum(b[2] for b in r[2]) if isinstance(r[2], (list, tuple)) else r[2] for r in requests]
        self.n = self.nv + np.array(nd, dtype=np.int32)
        self.T = self.ctx + self.n
        self.R = len(requests)
        self.q_indptr = np.concatenate([[0], np.cumsum(self.n)]).astype(np.int32)
        pages = (self.T + PAGE - 1) // PAGE + spare_pages_each
        self.page_indptr = np.concatenate([[0], np.cumsum(pages)]).astype(np.int32)
        self.num_pages = int(self.page_indptr[-1]) + spare
        self.page_indices = rng.permutation(self.num_pages)[:int(self.page_indptr[-1])].astype(np.int32)
        self.rows = int(self.q_indptr[-1])
        self.rng = rng

    def pages(self, r):
        return self.page_indices[self.page_indptr[r]:self.page_indptr[r + 1]]

    def places(self, r, count, first=0):
        """(pages, slots) of tokens first .. first + count - 1 of request r."""
        j = np.arange(first, first + count)
        return self.pages(r)[j // PAGE], j % PAGE

    def normal(self, *shape, std=1.0):
        return torch.from_numpy((self.rng.standard_normal(shape) * std).astype(np.float32)).to(torch.bfloat16)

    def q(self, std=1.0):
        return self.normal(self.rows, self.hq, self.d, std=std)

    def pool4(self, poison=0xff):
        """A 4-bit pool (numpy bytes): random codes and scales for every token
        that a request reads, `poison` everywhere else."""
        pool = np.full((self.num_pages, self.hkv, 17 * self.d), poison, dtype=np.uint8)
        code = [ref._code_places(self.d, kv) for kv in (0, 1)]
        scale = [ref._scale_places(self.d, kv) for kv in (0, 1)]
        for r in range(self.R):
            for p, page in enumerate(self.pages(r)):
                live = min(PAGE, int(self.T[r]) - PAGE * p) if self.n[r] else 0
                if live <= 0:
                    continue
                for kv in (0, 1):
                    for h in range(self.hkv):
                        pool[page, h][code[kv][:live]] = self.rng.integers(0, 256, (live, self.d // 2))
                        pool[page, h][scale[kv][:live]] = self.rng.integers(124, 128, (live, self.d // 32))
        return pool

    def branch_layout(self):
        flat = [b for one in self.branches for b in (one or [])]
        return binding.make_branches(np.concatenate([[0], np.cumsum([len(one or []) for one in self.branches])]),
                                     *([b[i] for b in flat] for i in range(3)))

    def device_pages(self, dev):
        return torch.as_tensor(self.page_indices, device=dev)

    def layout4(self, cache, ctx=None, **kw):
        return binding.make_kv4_layout(self.hq, cache, self.q_indptr, self.nv, self.ctx if ctx is None else ctx,
                                       self.page_indptr, self.device_pages(cache.device), **kw)

    def layout16(self, q, k_cache):
        return binding.make_layout(q, k_cache, self.q_indptr, self.nv, self.ctx, self.page_indptr,
                                   self.device_pages(q.device))

    # ---- 64-bit references
    def q_of(self, q, r, h):
        """q of request r's rows and KV head h: float64 [n, g, D]."""
        x = q[self.q_indptr[r]:self.q_indptr[r + 1], h * self.g:(h + 1) * self.g]
        return ref.bf16_values(W.bf16_bits(x))

    def keys_of(self, pool, r, h, T, kv=0):
        """K (or V) of request r's first T tokens: from bytes, or bf16 pools (K, V)."""
        if isinstance(pool, np.ndarray):
            return ref.tokens(pool, self.pages(r), h, T, kv)
        t = torch.from_numpy(self.pages(r).astype(np.int64))
        x = pool[kv][t, h]
        x = x.transpose(1, 2) if kv else x
        return ref.bf16_values(W.bf16_bits(x.reshape(-1, self.d)))[:T]

    def attention(self, q, pool, scale=None):
        """out, lse, and the weighted mean magnitude of V, [rows, Hq, ..]."""
        scale = self.d ** -0.5 if scale is None else scale
        out = np.zeros((self.rows, self.hq, self.d))
        lse, mag = np.zeros(out.shape[:2]), np.zeros(out.shape)
        for r in range(self.R):
            n = int(self.n[r])
            if n == 0:
                continue
            see = ref.visible(int(self.ctx[r]), int(self.nv[r]), n, self.branches[r])
            rows = slice(int(self.q_indptr[r]), int(self.q_indptr[r + 1]))
            for h in range(self.hkv):
                heads = slice(h * self.g, (h + 1) * self.g)
                T = int(self.T[r])
                out[rows, heads], lse[rows, heads], mag[rows, heads] = ref.attention(
                    self.q_of(q, r, h), self.keys_of(pool, r, h, T), self.keys_of(pool, r, h, T, 1), see, scale)
        return out, lse, mag

    def mass(self, old, q, pool, lse, count, decay, scale=None):
        """The mass pool after a call (numpy float64)."""
        scale = self.d ** -0.5 if scale is None else scale
        new = old.astype(np.float64).copy()
        for r in range(self.R):
            if self.n[r] == 0:
                continue
            L, V = int(self.ctx[r]), int(self.nv[r])
            page, slot = self.places(r, L + V)
            rows = slice(int(self.q_indptr[r]), int(self.q_indptr[r + 1]))
            for h in range(self.hkv):
                heads = slice(h * self.g, (h + 1) * self.g)
                new[page, h, slot] = ref.mass(new[page, h, slot], self.q_of(q, r, h), self.keys_of(pool, r, h, L + V),
                                              lse[rows, heads].astype(np.float64), L, V,
                                              None if count is None else int(count[r]), decay, scale)
        return new


def check_attention(out, lse, want, wlse, mag, score_size):
    """Element bounds.  The product takes each weight rounded to bf16 (2^-8 of
    the term) and the output is rounded once (2^-8 of it); 1 % of that and an
    absolute 1e-6 more cover the fp32 sums.  lse: fp32 dot products of D terms
    of total magnitude `score_size`, off by at most D 2^-24 of it, then a
    maximum, exponentials and a logarithm of a few ulps of values of that
    size."""
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    tol = 1.01 * 2.0 ** -8 * (mag + np.abs(want)) + 1e-6
    worst = np.max(np.abs(got - want) / tol)
    assert worst <= 1.0, f"output error {worst:.3f} of its bound"
    if lse is not None:
        err = np.abs(lse.double().cpu().numpy() - wlse).max()
        bound = (out.shape[-1] + 16) * 2.0 ** -24 * max(score_size, 1.0) + 1e-5
        assert err <= bound, f"lse error {err:.2e} > {bound:.2e}"
