"""Attention in training where the compiler spills: no more than it does (no GPU needed)."""
import re

from test_kernel_registers import metadata  # noqa: F401  (fixture)

# (kernel, width, rows straight to LDS): bytes of scratch, spilled vector registers, spilled scalar registers (into lanes of vector registers); others: none.
# Rows that are no multiples of 16 bytes come through registers, two tensors of up to 8 loads at once beside the accumulators.
MOST = {("self_forward", 128, 0): (112, 27, 11), ("self_query", 64, 0): (100, 24, 0), ("self_token", 64, 0): (36, 8, 15),
        ("self_forward", 96, 0): (0, 0, 31), ("self_query", 96, 0): (0, 0, 38), ("self_token", 96, 0): (0, 0, 76),
        ("self_query", 128, 0): (0, 0, 18), ("self_token", 128, 0): (0, 0, 50), ("self_token", 32, 0): (0, 0, 13),
        ("self_token", 32, 1): (0, 0, 4), ("self_token", 64, 1): (0, 0, 2), ("self_token", 96, 1): (0, 0, 6), ("self_token", 128, 1): (0, 0, 4)}


def test_attention_kernels_spill_no_more(metadata):  # noqa: F811
    seen = 0
    for name, k in metadata.items():
        m = re.search(r"(self_forward|self_query|self_token)_kernelILi(\d+)ELb([01])E", name)
        if m:
            seen += 1
            got = k[".private_segment_fixed_size"], k[".vgpr_spill_count"], k[".sgpr_spill_count"]
            most = MOST.get((m.group(1), int(m.group(2)), int(m.group(3))), (0, 0, 0))
            assert all(g <= x for g, x in zip(got, most)), (name, got, most)
    assert seen == 24
