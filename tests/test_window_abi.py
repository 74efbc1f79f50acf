"""Refusals of rotated appends, the 8-bit cache and attention over a window:
checked on the host before anything touches a device (no GPU)."""
import ctypes
import os

import pytest

from paper_2609_34388_amd import binding
from test_cache_abi import BAD_LAYOUTS, NULL, ODD, SHAPE, UNSUPPORTED, L, P

pytestmark = pytest.mark.skipif(not os.path.exists(binding.LIB_PATH), reason="library not built")


def lib():
    return binding.library()


def rotation(dims=128, interleaved=0, inv_freq=0x1000, positions=None):
    return ctypes.byref(binding.Rotation(dims, interleaved, inv_freq, positions))


def append(l, rot=None, q=P, qs=1024, q_out=P, k=P, ks=256, v=P, vs=256, kc=P, vc=P):
    a = lib().rg_kv_append(l.ref if l else None, rot, q, qs, q_out, k, ks, v, vs, kc, vc, None)
    b = lib().rg_kv8_append(l.ref if l else None, rot, q, qs, q_out, k, ks, v, vs, kc, vc, None)
    if vc is P:
        assert a == b
    return a


def read(l, cache=P, scales=P, k=P, ks=256, v=P, vs=256):
    return lib().rg_kv8_read(l.ref if l else None, cache, scales, k, ks, v, vs, None)


@pytest.mark.parametrize("call", [append, read])
def test_layout_refusals(call):
    assert call(None) == NULL
    for kw, want in BAD_LAYOUTS:
        assert call(L(**kw)) == want, kw


def test_append_refusals():
    for name in ("q", "q_out", "k", "v", "kc", "vc"):
        assert append(L(), **{name: None}) == NULL
        if name != "vc":
            assert append(L(), **{name: ODD}) == UNSUPPORTED
    # V pages want 16 bytes, scales four
    assert append(L(), vc=ODD) == UNSUPPORTED
    assert lib().rg_kv8_append(L().ref, None, None, 0, None, P, 256, P, 256, P, ctypes.c_void_p(0x1002), None) == UNSUPPORTED
    for name in ("ks", "vs"):
        assert append(L(), **{name: 248}) == SHAPE and append(L(), **{name: -256}) == SHAPE
        assert append(L(), **{name: 260}) == UNSUPPORTED
    assert append(L(), qs=1016) == SHAPE and append(L(), qs=1028) == UNSUPPORTED
    # in place only where rows lie behind one another
    assert append(L(), qs=1032) == SHAPE
    assert append(L(indices=0x1002)) == UNSUPPORTED


def test_rotation_refusals():
    assert append(L(), rot=rotation(inv_freq=None)) == NULL
    for dims in (-16, 8, 24, 144):
        assert append(L(), rot=rotation(dims=dims)) == SHAPE
    assert append(L(D=64), rot=rotation(dims=80)) == SHAPE
    assert append(L(), rot=rotation(inv_freq=0x1002)) == UNSUPPORTED
    assert append(L(), rot=rotation(positions=0x1001)) == UNSUPPORTED


def test_read_refusals():
    for name in ("k", "v", "cache", "scales"):
        assert read(L(), **{name: None}) == NULL
    for name in ("k", "v", "cache"):
        assert read(L(), **{name: ODD}) == UNSUPPORTED
    assert read(L(), scales=ctypes.c_void_p(0x1002)) == UNSUPPORTED
    assert read(L(), ks=248) == SHAPE and read(L(), vs=0) == SHAPE and read(L(), ks=257) == UNSUPPORTED


def window(size=10, sink=2):
    return ctypes.byref(binding.Window(size, sink))


def attend(l, w=None, q=P, cache=P, second=P, out=P, lse=None, ws=None, nbytes=0, br=None):
    ref, w = l.ref if l else None, window() if w is None else w
    a = lib().rg_kv8_attention(ref, br, w, q, cache, second, out, lse, ws, nbytes, None)
    b = lib().rg_window_attention(ref, br, w, q, cache, second, out, lse, ws, nbytes, None)
    if second is P:
        assert a == b
    return a


def test_attention_layout_refusals():
    assert attend(None) == NULL
    for kw, want in BAD_LAYOUTS:
        assert attend(L(**kw)) == want, kw


def test_attention_refusals():
    for name in ("q", "cache", "second", "out"):
        assert attend(L(), **{name: None}) == NULL
        if name != "second":
            assert attend(L(), **{name: ODD}) == UNSUPPORTED
    assert lib().rg_window_attention(L().ref, None, window(), P, P, ODD, P, None, None, 0, None) == UNSUPPORTED
    assert attend(L(), second=ctypes.c_void_p(0x1002)) == UNSUPPORTED
    assert attend(L(), lse=ctypes.c_void_p(0x1002)) == UNSUPPORTED
    assert attend(L(indices=0x1002)) == UNSUPPORTED
    for size, sink in ((0, 0), (-1, 5), (1, -1)):
        assert attend(L(), w=window(size, sink)) == SHAPE
    assert lib().rg_window_attention(L().ref, None, None, P, P, P, P, None, None, 0, None) == NULL
    long = L(ctx=(9000, 17))
    need = ctypes.c_size_t()
    query = lib().rg_kv8_attention_workspace
    assert query(long.ref, None, None, None) == NULL
    assert lib().rg_window_attention_workspace(long.ref, None, None, ctypes.byref(need)) == NULL
    assert query(long.ref, None, window(0), ctypes.byref(need)) == SHAPE
    assert query(long.ref, None, window(8000), ctypes.byref(need)) == 0 and need.value > 0
    few = window(8000)
    assert attend(long, few) == 4 and attend(long, few, ws=P, nbytes=need.value - 1) == 4
    assert attend(long, few, ws=ODD, nbytes=need.value) == 4
    all_keys = need.value
    assert query(long.ref, None, None, ctypes.byref(need)) == 0 and need.value >= all_keys
    br = binding.make_branches([0, 1, 2], [3, 0], [0, 0], [3, 5])
    assert attend(L(), br=ctypes.byref(br.c)) == SHAPE
    br.c.branch_indptr = None
    assert attend(L(), br=ctypes.byref(br.c)) == NULL


def test_sizes_past_32_bits():
    for size, sink in ((1 << 31, 0), ((1 << 32) + 5, 0), (5, 1 << 32), (-(1 << 32), 0)):
        with pytest.raises(ValueError):
            binding.make_window(size, sink)
    # a request's columns: rows x query heads of a KV head
    need = ctypes.c_size_t()
    for hq, want in ((16384, 0), (16640, UNSUPPORTED)):
        wide = L(n=(65535, 5), hq=hq, hkv=1)
        assert lib().rg_kv8_attention_workspace(wide.ref, None, None, ctypes.byref(need)) == want
        if want:
            assert attend(wide) == want


def test_windows_bound_the_workspace():
    """A window's keys, not the context's, are what is split."""
    need = ctypes.c_size_t()
    l = L(ctx=(900000, 17), pages=(60000, 2))
    for size in (1, 100):
        assert lib().rg_kv8_attention_workspace(l.ref, None, window(size, 4), ctypes.byref(need)) == 0
        assert need.value <= 4 << 20
    # the largest layouts and windows plan without overflow
    for w in (window(2 ** 31 - 1, 2 ** 31 - 1), window(1, 2 ** 31 - 1), None):
        far = L(ctx=(2 ** 30 - 8, 17), nv=(0, 5), pages=(1 << 26, 2))
        assert lib().rg_kv8_attention_workspace(far.ref, None, w, ctypes.byref(need)) == 0
