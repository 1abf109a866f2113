"""The kernels of attention in training, of rotary positions and of the optimizer's step keep their tiles in registers (no GPU needed)."""
import re

from test_kernel_registers import metadata  # noqa: F401  (fixture)


def test_training_kernels_keep_nothing_in_scratch(metadata):  # noqa: F811
    """Of attention those whose rows are loaded straight to LDS (heads of multiples of 8); of the others everything."""
    seen = []
    for name, k in metadata.items():
        m = re.search(r"(self_forward|self_query|self_token)_kernelILi(\d+)ELb1E|(self_join|rope|adamw_read|adamw)_kernel", name)
        if m:
            seen.append(m.group(1) or m.group(3))
            assert (k[".private_segment_fixed_size"], k[".vgpr_spill_count"]) == (0, 0), name
    assert [seen.count(x) for x in ("self_forward", "self_query", "self_token", "self_join", "rope", "adamw_read", "adamw")] == [4, 4, 4, 1, 8, 1, 12]
