"""What the compiler made of the attention kernels, and how large the decode workspace gets: no GPU needed."""
import ctypes as C
import re

import numpy as np
import pytest

from paper_2602_22592_amd import binding as pq
from test_kernel_registers import metadata  # noqa: F401  (fixture)


def test_kernels_keep_their_tiles_in_registers(metadata):  # noqa: F811
    """Every decode kernel, and those of prompts whose rows are shared by four wavefronts; heads beyond 128 run one wavefront a SIMD."""
    seen = set()
    for name, k in metadata.items():
        m = re.search(r"(attn_decode|attn_prefill|kv_write|kv_read)_kernel", name)
        if not m:
            continue
        seen.add(m.group(1))
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0, name
    assert seen == {"attn_decode", "attn_prefill", "kv_write", "kv_read"}


@pytest.mark.parametrize("seed", range(4))
def test_decode_workspace_holds_at_most_1024_pieces_a_row(seed):
    rng = np.random.default_rng(seed)
    for _ in range(200):
        d, Hk, G, page = int(rng.integers(1, 129)) * 2, int(rng.integers(1, 65)), int(rng.integers(1, 17)), 1 << int(rng.integers(4, 11))
        B, max_pages = int(rng.integers(0, 300)), int(rng.integers(1, (1 << 30) // page))
        kv = pq.make_kv_desc(int(rng.integers(0, 2)), Hk, d, page, 10, B, max_pages)
        a = pq.make_attn_desc(kv, Hk * G, window=int(rng.choice([0, 1, 5000, 2 ** 31 - 1])), max_len=int(rng.choice([0, 1, 70000, 2 ** 31 - 1])))
        n = pq.lib().pq_attn_decode_workspace_bytes(C.byref(a))
        row = B * Hk * G * (4 * (-(-d // 32) * 32) + 8)
        assert 256 <= n <= 1024 * row + 768
