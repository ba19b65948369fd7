"""Registers and spills of the kernels for many prompts (no GPU needed): what their launches rely on."""
import pytest

from test_kernel_resources import _resource_usage

# kernel, waves a SIMD at least, bytes of scratch a lane at most (many rows of 128 spill outside their loop over tiles where rows
# are 16-bit, and a few registers within it where they become bf16 on the way;
# 16 vectors of logits a thread spill three or four registers)
LIMITS = {
    "pages_attention.hip": [("few_pages_kernelILi128ELi16E", 2, 0), ("few_pages_kernelILi128ELi8E", 3, 0),
                            ("few_pages_kernelILi64E", 4, 0),
                            ("mixed_pages_kernelILi128ELi16E", 2, 96), ("mixed_pages_kernelILi128ELi8E", 2, 192),
                            ("mixed_pages_kernelILi64E", 2, 0), ("join_pages_kernel", 4, 0)],
    "pages_kernels.hip": [("pages_append_kernel", 8, 0), ("pages_read_kernel", 8, 0)],
    "rotate_kernels.hip": [("rotation_table_kernel", 4, 0), ("rotate_wide_kernel", 6, 0), ("rotate_rows_kernel", 5, 0), ("rotate_any_kernel", 8, 0)],
    "logprob_kernels.hip": [("logprob_kernelILb1ELi16E", 4, 16), ("logprob_kernelILb0ELi16E", 4, 16),
                            ("logprob_kernelILb1ELi8E", 4, 0), ("logprob_kernelILb0ELi8E", 4, 0), ("logprob_kernelILb1ELi4E", 8, 0),
                            ("logprob_kernelILb0ELi4E", 8, 0), ("logprob_kernelILb1ELi1E", 8, 0), ("logprob_kernelILb0ELi1E", 8, 0),
                            ("logprob_join_kernel", 8, 0)],
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
