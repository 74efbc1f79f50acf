"""Registers of the built attention kernels, from the code object's own notes
(no GPU): the kernels of the default launch mode keep everything in registers."""
import os
import re
import struct
import subprocess

import pytest

from paper_2609_34388_amd import binding

READELF = "/opt/rocm/llvm/bin/llvm-readelf"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"

pytestmark = pytest.mark.skipif(not (os.path.exists(binding.LIB_PATH) and os.path.exists(READELF)),
                                reason="library not built, or no llvm-readelf")


def _code_objects():
    """The gfx950 code objects bundled in the library, one per source file."""
    blob = open(binding.LIB_PATH, "rb").read()
    for at in (m.start() for m in re.finditer(MAGIC, blob)):
        count, pos = struct.unpack_from("<Q", blob, at + len(MAGIC))[0], at + len(MAGIC) + 8
        for _ in range(count):
            offset, size, idlen = struct.unpack_from("<QQQ", blob, pos)
            name = blob[pos + 24:pos + 24 + idlen].decode()
            pos += 24 + idlen
            if "gfx950" in name and size:
                yield blob[at + offset:at + offset + size]


def _kernels(tmp_path):
    """{kernel name: {note key: value}}"""
    out = {}
    for i, obj in enumerate(_code_objects()):
        path = tmp_path / f"{i}.co"
        path.write_bytes(obj)
        notes = subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True, check=True).stdout
        for block in notes.split("  - .agpr_count:")[1:]:
            got = dict(re.findall(r"^    \.(\w+): +(\S+)$", block, re.M))
            out[got["name"]] = got
    return out


def test_default_attention_kernels_do_not_spill(tmp_path):
    kernels = {k: v for k, v in _kernels(tmp_path).items() if "attn_fwd_kernel" in k or "attn_combine_kernel" in k}
    # head size x work group x plan form, and the merges of the two forms that split
    assert sum("attn_fwd_kernel" in k for k in kernels) == 2 * 2 * 3
    assert sum("attn_combine_kernel" in k for k in kernels) == 2 * 2 * 2
    for name, k in kernels.items():
        assert int(k["vgpr_spill_count"]) == 0 and int(k["private_segment_fixed_size"]) == 0, name
        assert int(k["vgpr_count"]) <= 168, name  # three waves per SIMD


@pytest.mark.parametrize("part, count, vgprs", [
    ("kv4_append_kernel", 2, 64), ("kv4_read_kernel", 2, 64),  # head sizes
    ("kv4_attn_kernel", 2 * 2, 256),                           # x plan forms; two waves per SIMD
    ("kv4_merge_kernel", 2 * 2 * 2, 128),                      # x threads of a row
    ("mass_kernel", 2 * 2, 168), ("mass_rows_kernel", 2 * 2, 168),  # x caches; three waves per SIMD
    ("evict_select_kernel", 4, 128),                           # slots of a thread; a work group of 1024 needs four
    ("evict_move_kernel", 2 * 2, 128)])
def test_cache_kernels_do_not_spill(tmp_path, part, count, vgprs):
    kernels = {k: v for k, v in _kernels(tmp_path).items() if part in k}
    assert len(kernels) == count
    for name, k in kernels.items():
        assert int(k["vgpr_spill_count"]) == 0 and int(k["private_segment_fixed_size"]) == 0, name
        assert int(k["vgpr_count"]) <= vgprs, name


def test_wide_mass_kernels_do_not_spill(tmp_path):
    kernels = {k: v for k, v in _kernels(tmp_path).items() if "mass_wide_kernel" in k}
    assert len(kernels) == 2 * 2  # head sizes x caches
    for name, k in kernels.items():
        assert int(k["vgpr_spill_count"]) == 0 and int(k["private_segment_fixed_size"]) == 0, name
        assert int(k["vgpr_count"]) <= 168, name  # three waves per SIMD


def test_eviction_choices_share_a_compute_unit(tmp_path):
    """Two work groups of 1024 on a compute unit leave 64 vector registers each;
    scalar registers that do not fit go to lanes of those, not to memory."""
    kernels = {k: v for k, v in _kernels(tmp_path).items() if "evict_select_kernel" in k}
    spills = {4: 0, 8: 16, 16: 64, 32: 140}  # by the held slots of a thread: their masks are two words each
    for held, most in spills.items():
        (k,) = [v for name, v in kernels.items() if f"evict_select_kernelILi{held}E" in name]
        assert int(k["vgpr_count"]) <= 64 and int(k["private_segment_fixed_size"]) == 0, held
        assert int(k["sgpr_spill_count"]) <= most, held


def test_scalar_spills_of_the_other_cache_kernels(tmp_path):
    parts = ("kv4_append", "kv4_read", "kv4_attn", "kv4_merge", "mass_kernel", "mass_wide", "mass_rows", "evict_move")
    for name, k in _kernels(tmp_path).items():
        if any(part in name for part in parts):
            # the attention's plan without branches: 20 words in lanes of a vector register
            assert int(k["sgpr_spill_count"]) <= (24 if "kv4_attn" in name else 0), name
