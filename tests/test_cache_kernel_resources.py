"""Registers and spills of the answering kernels (no GPU needed): what their launches rely on."""
import pytest

from test_kernel_resources import _resource_usage

# kernel, waves a SIMD at least, bytes of scratch a lane at most (where spilling a few registers was faster than fewer waves,
# or cost nothing that was measured)
LIMITS = {
    "cache_attention.hip": [("few_rows_kernelILi128E", 2, 0), ("few_rows_kernelILi64E", 3, 0), ("some_rows_kernel", 2, 0),
                            ("join_kernel", 4, 0), ("many_rows_kernel", 2, 0), ("weigh_some_kernel", 4, 0),
                            ("weigh_many_kernelILi128E", 3, 8), ("weigh_many_kernelILi64E", 3, 0)],
    "cache_kernels.hip": [("append_rows_kernel", 4, 0), ("append_columns_kernel", 4, 0), ("cache_read_kernel", 4, 0),
                          ("evict_select_kernel", 4, 0), ("evict_move_kernel", 4, 0)],
    "sample_kernels.hip": [("sample_max_kernel", 4, 0), ("sample_collect_kernel", 4, 0), ("sample_kernelItLb", 4, 0),
                           ("sample_kernelIfLb0E", 4, 20), ("sample_kernelIfLb1E", 4, 0)],
}


@pytest.mark.parametrize("src", sorted(LIMITS))
def test_waves_and_spills(src):
    kernels = _resource_usage(src)
    seen = set()
    for part, waves, scratch in LIMITS[src]:
        found = {n: v for n, v in kernels.items() if part in n}
        assert found, part
        seen |= set(found)
        for name, v in found.items():
            assert v["Occupancy"] >= waves and v["ScratchSize"] <= scratch, (name, v)
    assert seen == {n for n, v in kernels.items() if "ScratchSize" in v}      # (none is left out)
