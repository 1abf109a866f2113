"""What the cache and attention calls refuse, on the host, before anything is launched (no GPU needed)."""
import ctypes as C
import os

import pytest
import torch

from paper_2602_22592_amd import binding as pq

I8, BF = pq.PQ_KV_INT8, pq.PQ_KV_BF16
fake, big = C.c_void_p(0x1000), C.c_size_t(1 << 50)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pq.LIB_PATH):
        from paper_2602_22592_amd.build import build
        build(verbose=False)
    return pq.lib()


def kv(kind=I8, Hk=2, d=64, page=16, n_pages=8, B=2, max_pages=4):
    return pq.make_kv_desc(kind, Hk, d, page, n_pages, B, max_pages)


def test_cache_sizes(lib):
    size = lambda **k: lib.pq_kv_cache_bytes(C.byref(kv(**k)))
    assert size() == 8 * 2 * (2 * 16 * 64 + 8 * 16)
    assert size(kind=BF, d=90, page=128) == 8 * 2 * (2 * 128 * 96 * 2)
    assert size(n_pages=1 << 20, page=1024, d=256) == (1 << 20) * 2 * (2 * 1024 * 256 + 8 * 1024)      # beyond 32 bits


@pytest.mark.parametrize("bad,code", [(dict(kind=2), -1), (dict(Hk=0), -1), (dict(d=63), -2), (dict(d=258), -2), (dict(d=0), -1), (dict(page=8), -2),
                                      (dict(page=48), -2), (dict(page=2048), -2), (dict(n_pages=0), -1), (dict(B=-1), -1), (dict(max_pages=0), -1),
                                      (dict(max_pages=1 << 27), -2), (dict(Hk=70000), -2)])
def test_bad_descriptors(lib, bad, code):
    d = kv(**bad)
    assert lib.pq_kv_cache_bytes(C.byref(d)) == 0
    assert lib.pq_kv_write(C.byref(d), fake, fake, 1, 4, C.c_int64(128), C.c_int64(128), None, fake, fake, fake, big, None) == code
    a = pq.make_attn_desc(d, max(d.n_kv_heads, 1) * 2, scale=1.0)
    assert lib.pq_attn_decode_workspace_bytes(C.byref(a)) == 0
    assert lib.pq_attn_decode(C.byref(a), fake, C.c_int64(256), fake, big, fake, fake, fake, None, fake, big, None) == code
    assert lib.pq_attn_prefill(C.byref(a), fake, C.c_int64(256), 4, fake, fake, big, fake, fake, fake, None, None) == code


def test_bad_cache_calls(lib):
    d = kv()

    def write(K=fake, V=fake, dtype=1, T=4, ks=128, vs=128, lens=fake, table=fake, cache=fake, size=big, desc=d):
        return lib.pq_kv_write(C.byref(desc), K, V, dtype, T, C.c_int64(ks), C.c_int64(vs), None, lens, table, cache, size, None)

    def read(K=fake, V=fake, dtype=1, T=4, ks=128, vs=128, lens=fake, table=fake, cache=fake, size=big, desc=d):
        return lib.pq_kv_read(C.byref(desc), cache, size, None, lens, table, T, K, V, dtype, C.c_int64(ks), C.c_int64(vs), None)

    odd = C.c_void_p(0x1008)
    for f in (write, read):
        assert f(dtype=5) == -3 and f(T=-1) == -1 and f(lens=None) == -1 and f(table=None) == -1 and f(cache=None) == -1
        assert f(ks=126) == -2 and f(vs=129) == -2 and f(K=odd) == -2 and f(V=odd) == -2 and f(cache=odd) == -2
        assert f(size=C.c_size_t(lib.pq_kv_cache_bytes(C.byref(d)) - 1)) == -4
        assert f(T=0) == 0 and f(desc=kv(B=0)) == 0                       # nothing to do: nothing launched
        assert f(desc=kv(Hk=60000, d=2), T=0x7fffffff, ks=120000, vs=120000) == -2
    assert write(K=None) == -1 and write(V=None) == -1 and read(K=None, V=None) == -1


def test_bad_attention_calls(lib):
    def desc(heads=4, causal=True, window=0, max_len=0, scale=1.0, **k):
        return pq.make_attn_desc(kv(**k), heads, scale=scale, causal=causal, window=window, max_len=max_len)

    def decode(a, Q=fake, qs=256, cache=fake, size=big, lens=fake, table=fake, O=fake, ws=fake, wsize=big):
        return lib.pq_attn_decode(C.byref(a), Q, C.c_int64(qs), cache, size, lens, table, O, None, ws, wsize, None)

    def prefill(a, Q=fake, qs=256, cache=fake, size=big, lens=fake, table=fake, O=fake, T=4):
        return lib.pq_attn_prefill(C.byref(a), Q, C.c_int64(qs), T, None, cache, size, lens, table, O, None, None)

    odd = C.c_void_p(0x1008)
    for f in (decode, prefill):
        for bad in (dict(heads=3), dict(heads=0), dict(window=-1), dict(max_len=-1), dict(scale=float("nan")), dict(scale=float("inf")),
                    dict(causal=False, window=3)):
            assert f(desc(**bad)) == -1
        a = desc()
        assert f(a, Q=None) == -1 and f(a, O=None) == -1 and f(a, cache=None) == -1 and f(a, lens=None) == -1 and f(a, table=None) == -1
        assert f(a, qs=254) == -2 and f(a, qs=257) == -2 and f(a, Q=odd) == -2 and f(a, O=odd) == -2 and f(a, cache=odd) == -2
        assert f(a, size=C.c_size_t(lib.pq_kv_cache_bytes(C.byref(a.kv)) - 1)) == -4
        assert f(desc(B=0)) == 0
    a = desc(max_len=5000, max_pages=1000)
    need = lib.pq_attn_decode_workspace_bytes(C.byref(a))
    assert need > 0 and decode(a, wsize=C.c_size_t(need - 1)) == -4 and decode(a, ws=None) == -1 and decode(a, ws=odd) == -2
    assert prefill(desc(), T=-1) == -1 and prefill(desc(), T=0) == 0
    assert prefill(desc(heads=4000, Hk=2000), qs=4000 * 64, T=0x7fffffff) == -2


def test_the_binding_refuses_tensors_that_do_not_fit():
    """Shapes, types, strides and devices, checked before the library is called."""
    d = kv()
    a = pq.make_attn_desc(d, 4)
    cache = torch.zeros(pq.lib().pq_kv_cache_bytes(C.byref(d)), dtype=torch.uint8)
    lens, table = torch.zeros(2, dtype=torch.int32), torch.zeros((2, 4), dtype=torch.int32)
    K = torch.zeros((2, 2, 64))
    with pytest.raises(pq.PQError, match="GPU"):                          # host tensors
        pq.kv_write(d, K, K, cache, lens, table)
    with pytest.raises(pq.PQError, match="int32"):
        pq.kv_write(d, K, K, cache, lens.long(), table)
    with pytest.raises(pq.PQError, match="rows, 2, 64"):
        pq._rows(torch.zeros(2, 128), 2, 64)
    with pytest.raises(pq.PQError, match="contiguous"):
        pq._rows(torch.zeros(2, 2, 128)[..., ::2], 2, 64)
    with pytest.raises(pq.PQError, match="contiguous"):
        pq._rows(torch.zeros(2, 64, 2).transpose(1, 2), 2, 64)
    assert pq._rows(torch.zeros(5, 4, 64)[:, 1:3], 2, 64) == (5, 256) and pq._rows(torch.zeros(1, 2, 64), 2, 64) == (1, 128)
    Q = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    for bad in (dict(Q=Q.float()), dict(O=Q.float()), dict(O=Q[:1]), dict(lse=torch.zeros(7)), dict(lse=torch.zeros(8, dtype=torch.float64))):
        with pytest.raises(pq.PQError):
            pq._attn_rows(a, **{**dict(Q=Q, O=Q, lse=None), **bad})
    with pytest.raises(pq.PQError, match="descriptor"):
        pq.kv_cache(kv(d=63))
    with pytest.raises(pq.PQError, match="descriptor"):
        pq.attn_decode_workspace(pq.make_attn_desc(kv(), 3))
