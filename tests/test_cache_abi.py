"""Refusals of the 4-bit cache, mass and eviction calls: checked on the host
before anything touches a device (no GPU)."""
import ctypes
import os

import numpy as np
import pytest

from paper_2609_34388_amd import binding

pytestmark = pytest.mark.skipif(not os.path.exists(binding.LIB_PATH), reason="library not built")
P = ctypes.c_void_p(0x1000)  # never dereferenced on these paths
ODD = ctypes.c_void_p(0x1004)
NULL, SHAPE, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4


class L:
    def __init__(self, ctx=(40, 17), nv=(3, 0), n=(7, 5), hq=8, hkv=2, D=128, page=16, pages=None, indices=0x1000):
        self.q = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        self.nv, self.ctx = np.array(nv, np.int32), np.array(ctx, np.int32)
        pages = [(c + k + 15) // 16 for c, k in zip(ctx, n)] if pages is None else pages
        self.pi = np.concatenate([[0], np.cumsum(pages)]).astype(np.int32)
        self.c = binding.AttnLayout(len(ctx), hq, hkv, D, page, 64, 0.0, self.q.ctypes.data, self.nv.ctypes.data,
                                    self.ctx.ctypes.data, self.pi.ctypes.data, indices)
        self.ref = ctypes.byref(self.c)


class E:
    def __init__(self, ctx=(100, 64), keep=(50, 64), tracked=(0, 0), evicted=(0, 0), hkv=2, D=128, page=16, sink=4,
                 recent=8, pages=None):
        i = lambda x: np.array(x, np.int32)
        self.a = [i(ctx), i(keep), i(tracked), i(evicted),
                  i(np.concatenate([[0], np.cumsum([(c + 15) // 16 for c in ctx] if pages is None else pages)]))]
        self.c = binding.EvictLayout(len(ctx), hkv, D, page, 64, sink, recent, *(x.ctypes.data for x in self.a),
                                     P.value)
        self.ref = ctypes.byref(self.c)


def lib():
    return binding.library()


def append(l, k=P, ks=256, v=P, vs=256, cache=P):
    return lib().rg_kv4_append(l.ref if l else None, k, ks, v, vs, cache, None)


def read(l, cache=P, k=P, ks=256, v=P, vs=256):
    return lib().rg_kv4_read(l.ref if l else None, cache, k, ks, v, vs, None)


def attend(l, q=P, cache=P, out=P, lse=None, ws=None, nbytes=0, br=None):
    return lib().rg_kv4_attention(l.ref if l else None, br, q, cache, out, lse, ws, nbytes, None)


def mass(l, q=P, k=P, lse=P, count=None, decay=1.0, m=P):
    a = lib().rg_attention_mass(l.ref if l else None, q, k, lse, count, decay, m, None)
    b = lib().rg_kv4_attention_mass(l.ref if l else None, q, k, lse, count, decay, m, None)
    assert a == b
    return a


def evict(l, k=P, v=P, score=P, m=None, pos=P, ws=P, nbytes=1 << 30):
    a = lib().rg_evict_tokens(l.ref if l else None, k, v, score, m, pos, ws, nbytes, None)
    if v is P:
        b = lib().rg_kv4_evict_tokens(l.ref if l else None, k, score, m, pos, ws, nbytes, None)
        assert a == b
    return a


BAD_LAYOUTS = [(dict(D=96), UNSUPPORTED), (dict(page=32), UNSUPPORTED), (dict(hq=6, hkv=4), SHAPE),
               (dict(nv=(8, 0)), SHAPE), (dict(ctx=(-1, 3)), SHAPE), (dict(pages=(2, 2)), SHAPE),
               (dict(n=(70000, 5), nv=(0, 0)), UNSUPPORTED), (dict(hkv=0), SHAPE)]


@pytest.mark.parametrize("call", [append, read, attend, mass])
def test_layout_refusals(call):
    assert call(None) == NULL
    for kw, want in BAD_LAYOUTS:
        assert call(L(**kw)) == want, kw


def test_row_refusals():
    for call in (append, read):
        for name in ("k", "v", "cache"):
            assert call(L(), **{name: None}) == NULL
            assert call(L(), **{name: ODD}) == UNSUPPORTED
        assert call(L(), ks=248) == SHAPE and call(L(), vs=0) == SHAPE and call(L(), ks=-256) == SHAPE
        assert call(L(), ks=257) == UNSUPPORTED and call(L(), vs=260) == UNSUPPORTED


def test_attention_refusals():
    for name in ("q", "cache", "out"):
        assert attend(L(), **{name: None}) == NULL
        assert attend(L(), **{name: ODD}) == UNSUPPORTED
    assert attend(L(indices=0x1002)) == UNSUPPORTED
    long = L(ctx=(9000, 17))
    need = ctypes.c_size_t()
    assert lib().rg_kv4_attention_workspace(long.ref, None, ctypes.byref(need)) == 0 and need.value > 0
    assert attend(long) == WORKSPACE and attend(long, ws=P, nbytes=need.value - 1) == WORKSPACE
    assert attend(long, ws=ODD, nbytes=need.value) == WORKSPACE
    assert lib().rg_kv4_attention_workspace(long.ref, None, None) == NULL
    # branches: rows that do not add up, and a missing list
    br = binding.make_branches([0, 1, 2], [3, 0], [0, 0], [3, 5])
    assert attend(L(), br=ctypes.byref(br.c)) == SHAPE
    br.c.branch_indptr = None
    assert attend(L(), br=ctypes.byref(br.c)) == NULL


def test_mass_refusals():
    for name in ("q", "k", "lse", "m"):
        assert mass(L(), **{name: None}) == NULL
    assert mass(L(), q=ODD) == UNSUPPORTED and mass(L(), k=ODD) == UNSUPPORTED
    assert mass(L(), m=ctypes.c_void_p(0x1002)) == UNSUPPORTED
    for decay in (-0.5, float("nan"), float("inf")):
        assert mass(L(), decay=decay) == SHAPE


def test_evict_refusals():
    assert evict(None) == NULL
    for name in ("k", "v", "score", "pos"):
        assert evict(E(), **{name: None}) == NULL
    assert evict(E(), k=ODD) == UNSUPPORTED and evict(E(), v=ODD) == UNSUPPORTED
    assert evict(E(), score=ctypes.c_void_p(0x1002)) == UNSUPPORTED
    for kw, want in [(dict(D=96), UNSUPPORTED), (dict(page=8), UNSUPPORTED), (dict(hkv=0), SHAPE),
                     (dict(ctx=(-1, 64)), SHAPE), (dict(keep=(-1, 64)), SHAPE), (dict(tracked=(101, 0)), SHAPE),
                     (dict(tracked=(-1, 0)), SHAPE), (dict(evicted=(0, -1)), SHAPE), (dict(pages=(6, 4)), SHAPE),
                     (dict(sink=-1), SHAPE), (dict(recent=-1), SHAPE),
                     (dict(keep=(11, 64)), SHAPE),  # room for fewer than the 12 protected tokens
                     (dict(evicted=(2 ** 31 - 50, 0)), UNSUPPORTED)]:
        assert evict(E(**kw)) == want, kw
    need = ctypes.c_size_t()
    assert lib().rg_evict_workspace(E().ref, ctypes.byref(need)) == 0 and need.value > 0
    assert lib().rg_evict_workspace(E().ref, None) == NULL
    assert evict(E(), ws=None) == WORKSPACE and evict(E(), nbytes=need.value - 1) == WORKSPACE
    assert evict(E(), ws=ODD, nbytes=need.value) == WORKSPACE


def test_keep_below_the_protected_is_fine_where_nothing_is_cut():
    n = ctypes.c_size_t()
    assert lib().rg_evict_workspace(E(ctx=(10, 64), keep=(11, 64)).ref, ctypes.byref(n)) == 0


def test_mass_of_more_query_bytes_than_offsets_hold():
    """A request's verify rows of q must span less than 2^31 bytes where the
    kernel of many columns takes them."""
    for hq, want in ((256, UNSUPPORTED), (128, None)):
        l = L(ctx=(0,), nv=(65535,), n=(65535,), hq=hq, hkv=hq)
        # group 1: more than 128 columns either way; the smaller one is refused for its alignment alone
        assert mass(l, m=ctypes.c_void_p(0x1002)) == UNSUPPORTED
        if want:
            assert mass(l) == want


def test_mass_refuses_before_it_launches():
    """A batch of both kinds of requests one of whose launches is too large."""
    n = 1 << 14
    l = L(ctx=(1 << 29, 0), nv=(1, 200), n=(1, 200), hq=n, hkv=n)
    assert mass(l) == UNSUPPORTED
    l = L(ctx=(40, 1 << 29), nv=(1, 200), n=(1, 200), hq=n, hkv=n, D=64)
    assert mass(l) == UNSUPPORTED


@pytest.mark.parametrize("call", [append, read])
def test_rows_check_the_whole_layout(call):
    """Fields that rows do not use have to be valid all the same."""
    null = ctypes.c_void_p(None)
    assert call(L(nv=(7, 5), hq=2), cache=null) == NULL and call(L(nv=(0, 0), hq=64), cache=null) == NULL
    for kw in (dict(nv=(8, 0)), dict(nv=(0, -1)), dict(hq=3), dict(hq=0)):
        assert call(L(**kw), cache=null) == SHAPE, kw


@pytest.mark.parametrize("n, hq, D, fits", [(65535, 128, 128, True), (65535, 129, 128, False), (32767, 256, 128, True),
                                            (32768, 256, 128, False), (65535, 256, 64, True), (65535, 257, 64, False),
                                            (100, 8, 128, True)])
def test_mass_bound_of_query_bytes_from_both_sides(n, hq, D, fits):
    """Of a layout alone, before any pointer: one that fits goes on to the
    missing pointer.  The largest byte that fits is 2^31 - 32768."""
    assert (n * hq * D * 2 < 2 ** 31) == fits
    for hkv in {1, hq}:
        assert mass(L(ctx=(0,), nv=(n,), n=(n,), hq=hq, hkv=hkv, D=D), m=None) == (NULL if fits else UNSUPPORTED)
    # draft rows do not count
    assert mass(L(ctx=(0,), nv=(1,), n=(65535,), hq=1 << 12, hkv=1, D=D), m=None) == NULL
