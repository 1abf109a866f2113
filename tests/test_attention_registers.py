"""The kernels of short prompts, of 16-bit heads beyond 128 and of the joins keep their tiles in registers as well (no GPU needed)."""
import re

from test_kernel_registers import metadata  # noqa: F401  (fixture)


def test_kernels_of_few_rows_and_joins_keep_nothing_in_scratch(metadata):  # noqa: F811
    """Every type and width: eight blocks of 32 elements in both types, and one kernel that joins."""
    seen = []
    for name, k in metadata.items():
        m = re.search(r"(attn_rows|attn_join)_kernel", name)
        if m:
            seen.append(m.group(1))
            assert (k[".private_segment_fixed_size"], k[".vgpr_spill_count"]) == (0, 0), name
    assert seen.count("attn_rows") == 16 and seen.count("attn_join") == 1
