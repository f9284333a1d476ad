"""Registers, LDS and scratch memory of the prompt-side kernels, as the compiler recorded them (no GPU needed)."""
import pytest

from test_kernel_resources import _kernels


@pytest.fixture(scope="module")
def kernels():
    return _kernels()


@pytest.mark.parametrize("part", ["rope_kernel", "chunk_rows_kernel", "chunk_tokens_kernel", "join_tokens_kernel",
                                  "join_rows_kernel", "mass_kernel", "mass_split_kernel", "evict_select_kernel", "evict_count_kernel",
                                  "evict_collect_kernel", "evict_place_kernel", "evict_rows_kernel"])
def test_no_scratch_memory(kernels, part):
    some = {n: k for n, k in kernels.items() if part in n}
    assert some
    bad = {n: (k[".vgpr_spill_count"], k[".private_segment_fixed_size"]) for n, k in some.items()
           if k[".vgpr_spill_count"] or k[".private_segment_fixed_size"]}
    assert not bad


def test_two_attention_workgroups_share_a_compute_unit(kernels):
    # 2 x 4 wavefronts on 4 SIMDs of 512 registers, 160 KB of LDS; the loads into LDS address its first 64 KB, which the tiles
    # are, so that what follows them may not grow in front
    some = {n: k for n, k in kernels.items() if "chunk_rows_kernel" in n or "chunk_tokens_kernel" in n}
    assert len(some) == 16
    assert all(k[".vgpr_count"] <= 256 and 65536 <= k[".group_segment_fixed_size"] <= 80 * 1024 for k in some.values())


def test_two_weight_workgroups_share_a_compute_unit(kernels):
    some = {n: k for n, k in kernels.items() if "mass_kernel" in n}
    assert len(some) == 2
    assert all(k[".max_flat_workgroup_size"] == 512 and k[".vgpr_count"] <= 128 and
               k[".group_segment_fixed_size"] <= 80 * 1024 for k in some.values())
