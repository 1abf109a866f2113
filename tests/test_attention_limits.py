"""Limits of the cache and attention calls that the host decides (no GPU needed)."""
import ctypes as C

import pytest

from paper_2602_22592_amd import binding as pq
from test_attention_refusals import BF, big, fake, kv, lib  # noqa: F401  (lib: fixture)


@pytest.mark.parametrize("Hk,n_pages", [(32768, 2 ** 29 + 1), (65535, 2 ** 31 - 1), (32768, 2 ** 28)])
def test_caches_whose_size_passes_64_bits_are_refused(lib, Hk, n_pages):  # noqa: F811
    """A page of 2^20 bytes a head: 2^15 heads and 2^29 + 1 pages are 2^64 + 2^35 bytes, of which a size held in 64 bits keeps 2^35."""
    d = kv(kind=BF, Hk=Hk, d=256, page=1024, n_pages=n_pages)
    assert lib.pq_kv_cache_bytes(C.byref(d)) == 0
    row = C.c_int64(Hk * 256)
    assert lib.pq_kv_write(C.byref(d), fake, fake, 1, 4, row, row, None, fake, fake, fake, big, None) == -2
    a = pq.make_attn_desc(d, Hk)
    assert lib.pq_attn_decode_workspace_bytes(C.byref(a)) == 0
    assert lib.pq_attn_prefill(C.byref(a), fake, row, 4, fake, fake, big, fake, fake, fake, None, None) == -2


def test_the_largest_cache_is_counted_whole(lib):  # noqa: F811
    d = kv(kind=BF, Hk=32768, d=256, page=1024, n_pages=2 ** 27)
    assert lib.pq_kv_cache_bytes(C.byref(d)) == 2 ** 62
