"""Registers of the built kernels of rotated appends, the 8-bit cache and windowed
attention, from the code object's own notes (no GPU): nothing goes to memory."""
import pytest

from test_kernel_resources import _kernels, pytestmark  # noqa: F401


@pytest.mark.parametrize("part, count, vgprs", [
    ("13append_kernel", 2 * 2 * 2, 128),                       # head sizes x caches x pairs; four waves per SIMD
    ("kv8_read_kernel", 2, 64),                                # head sizes; eight
    ("kv8_attn_kernelILi128", 2, 256),                         # plan forms; two
    ("kv8_attn_kernelILi64", 2, 168),                          # three
    ("window_attn_kernel", 2 * 2, 256),                        # head sizes x plan forms; two
    ("window_merge_kernel", 2 * 2 * 2, 128)])                  # x waves of a row
def test_window_kernels_do_not_spill(tmp_path, part, count, vgprs):
    kernels = {k: v for k, v in _kernels(tmp_path).items() if part in k}
    assert len(kernels) == count
    for name, k in kernels.items():
        assert int(k["vgpr_spill_count"]) == 0 and int(k["private_segment_fixed_size"]) == 0, name
        assert int(k["vgpr_count"]) <= vgprs, name
