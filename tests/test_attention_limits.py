"""Limits of the cache and attention calls that the host decides (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2602_22592_amd import binding as pq
from paper_2602_22592_amd.stack import CachedAttention
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


def test_the_layer_refuses_weights_and_rows_that_do_not_fit():
    """Before anything is packed or launched: heads that do not divide the width, weights of another shape, rows that are not contiguous."""
    W = {"W" + n: torch.zeros((512 if n in "qo" else 128, 512), dtype=torch.bfloat16) for n in "qkvo"}
    pages = dict(n_pages=4, n_seqs=2, max_pages=2, device="cpu")
    for heads, kv_heads in ((7, 1), (12, 4), (8, 3), (0, 1), (8, 0)):
        with pytest.raises(pq.PQError, match="multiple of n_heads"):
            CachedAttention(W, heads, kv_heads, **pages)
    with pytest.raises(pq.PQError, match="Wk of shape"):
        CachedAttention(W, 8, 4, **pages)                                 # (its keys have 256 elements, not 128)
    with pytest.raises(pq.PQError, match="Wo of shape"):
        CachedAttention({**W, "Wo": W["Wo"].t()}, 8, 2, **pages)
    layer = CachedAttention.__new__(CachedAttention)
    layer.d, layer.B, layer.cache = 512, 2, torch.zeros(256, dtype=torch.uint8)
    x = torch.zeros((2, 512), dtype=torch.bfloat16)
    for bad in (torch.zeros((2, 1024), dtype=torch.bfloat16)[:, ::2], x.float(), x[:1], torch.zeros((512, 2), dtype=torch.bfloat16).t(), x[0]):
        for call in (lambda: layer.token(bad, None, None, x), lambda: layer.token(x, None, None, bad)):
            layer.step = {}
            with pytest.raises(pq.PQError, match="is wanted"):
                call()
    for bad in (torch.zeros((9, 1024), dtype=torch.bfloat16)[:, :512], x.float(), x[0], x[0, 0]):
        with pytest.raises(pq.PQError, match="is wanted"):
            layer.prompt(bad, None, None, None)


def test_the_layer_refuses_weights_that_are_not_on_one_gpu():
    W = {"W" + n: torch.zeros((512 if n in "qo" else 128, 512), dtype=torch.bfloat16) for n in "qkvo"}
    for device in ("cpu", "cuda", "cuda:1"):
        with pytest.raises(pq.PQError, match="one GPU"):
            CachedAttention(W, 8, 2, n_pages=4, n_seqs=2, max_pages=2, device=device)


def test_the_layer_runs_on_its_caches_device_whichever_is_current(monkeypatch):
    """Every call of a prompt and of a token finds the cache's device current (here -1, the host's number) though another one, 3, was."""
    current, found = [3], []

    class Device:
        def __init__(self, device):
            self.number = -1 if device == torch.device("cpu") else None

        def __enter__(self):
            self.before, current[0] = current[0], self.number

        def __exit__(self, *_):
            current[0] = self.before

    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(pq, "_current_device", lambda: current[0])
    monkeypatch.setattr(pq, "LinearBuffers", lambda *a: None)
    for name, out in (("linear_fwd", 3), ("decode_gemv", 4), ("kv_write", 3), ("attn_prefill", 6), ("attn_decode", 5), ("glue_lincomb", 0)):
        monkeypatch.setattr(pq, name, lambda *a, name=name, out=out, **k: (found.append((name, current[0])), a[out])[1])
    layer = CachedAttention.__new__(CachedAttention)
    layer.d, layer.B, layer.H, layer.Hk, layer.dh, layer.cache = 64, 2, 2, 1, 32, torch.zeros(256, dtype=torch.uint8)
    layer.kv = layer.attn = layer.attn_ws = None
    layer.packed = {n: (64 if n in "qo" else 32, None, None, None, None) for n in "qkvo"}
    layer.step = {n: torch.zeros((2, p[0]), dtype=torch.bfloat16) for n, p in layer.packed.items()}
    layer.step["a"] = torch.zeros((2, 64), dtype=torch.bfloat16)
    layer.decode = layer.decode_ws = {n: None for n in "qkvo"}
    x = torch.zeros((2, 64), dtype=torch.bfloat16)
    layer.prompt(x, None, None, None)
    layer.token(x, None, None, x.clone())
    assert len(found) == 14 and {number for _, number in found} == {-1} and current == [3]


def test_page_tables_of_another_width_are_refused():
    """A table with more entries a row than the descriptor says is large enough, but its rows lie elsewhere."""
    d = kv()
    cache, lens = torch.zeros(pq.lib().pq_kv_cache_bytes(C.byref(d)), dtype=torch.uint8), torch.zeros(2, dtype=torch.int32)
    table = lambda *shape: torch.zeros(shape, dtype=torch.int32)
    for shape in ((2, 8), (4, 2), (8, 1)):
        with pytest.raises(pq.PQError, match="4 in the descriptor"):
            pq._kv_check(d, cache, lens, table(*shape), None)
    for shape in ((2, 4), (3, 4), (8,), (20,)):                           # (what remains wrong with these is that they are host tensors)
        with pytest.raises(pq.PQError, match="on a GPU"):
            pq._kv_check(d, cache, lens, table(*shape), None)
    with pytest.raises(pq.PQError, match="on a GPU"):
        pq._kv_check(kv(B=1), cache, lens, table(1, 9), None)            # (one row)
