"""The paged key-value cache: what pq_kv_write leaves in memory, bit for bit, and what pq_kv_read makes of it."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from paged_cases import Paged, padded
from paper_2602_22592_amd import binding as pq

pytestmark = pytest.mark.gpu
BF, I8 = pq.PQ_KV_BF16, pq.PQ_KV_INT8


def raw_views(desc, raw):
    """Keys, values, key steps, value steps of a cache's bytes (numpy), as the header lays them out."""
    i8 = desc.kv_kind == I8
    dp, page = padded(desc.d_head), desc.page_tokens
    part = page * dp * (1 if i8 else 2)
    v = raw.reshape(desc.n_pages, desc.n_kv_heads, -1)
    assert v.shape[-1] == 2 * part + (8 * page if i8 else 0)
    cut = lambda a, b, t: np.ascontiguousarray(v[..., a:b]).view(t)
    t = np.int8 if i8 else np.uint16
    keys = cut(0, part, t).reshape(desc.n_pages, desc.n_kv_heads, page, dp)
    values = cut(part, 2 * part, t).reshape(desc.n_pages, desc.n_kv_heads, page // 16, dp, 16)
    steps = [cut(2 * part + 4 * page * i, 2 * part + 4 * page * (i + 1), np.uint32) if i8 else None for i in (0, 1)]
    return keys, values, steps[0], steps[1]


def as_codes(x, i8):
    """(stored numbers, steps) of rows x [n][Hk][d]."""
    if i8:
        c, s = ao.quantise(x)
        return c, s.view(np.uint32)
    return (ao.bf16(x).view(np.uint32) >> 16).astype(np.uint16), None


def write_case(kind, dtype, lens, rows, Hk, d, page, seed, extra=0, gap=0):
    """Writes the last rows[b] tokens of each sequence into a cache full of 0xff and returns everything to compare with."""
    c = Paged(kind, lens, Hk, d, page, seed)
    rng = np.random.default_rng(seed + 1)
    T = sum(rows)
    width = Hk * d + gap
    full = [torch.from_numpy(rng.standard_normal((T + extra, width)).astype(np.float32) * 3).to(dtype).cuda() for _ in range(2)]
    K, V = (x[:, :Hk * d].unflatten(1, (Hk, d)) for x in full)
    desc = c.desc()
    cache = pq.kv_cache(desc)
    cache.fill_(255)
    t32 = lambda a: torch.tensor(a, dtype=torch.int32).cuda()
    starts = t32(np.concatenate([[0], np.cumsum(rows)]))
    dev = (t32(lens), torch.from_numpy(c.table).cuda())
    pq.kv_write(desc, K, V, cache, *dev, row_start=starts)
    torch.cuda.synchronize()
    return c, desc, K, V, cache, dev, starts


SHAPES = [  # lens, rows, Hk, d, page
    ([1], [1], 1, 64, 16), ([5, 17, 1, 40], [5, 17, 1, 40], 3, 64, 16), ([33, 100, 16], [2, 37, 16], 4, 90, 32),
    ([7, 0, 64, 300], [3, 0, 1, 300], 2, 128, 128), ([50, 31], [33, 31], 5, 30, 16), ([129], [128], 2, 256, 64),
    ([20, 20, 20], [1, 1, 1], 16, 64, 16), ([70], [70], 1, 2, 16), ([90, 47], [61, 30], 2, 96, 64), ([2000, 3], [1987, 3], 2, 80, 16),
]


@pytest.mark.parametrize("kind,dtype", [(I8, torch.bfloat16), (I8, torch.float32), (BF, torch.bfloat16), (BF, torch.float32)])
@pytest.mark.parametrize("lens,rows,Hk,d,page", SHAPES)
def test_write_is_bit_exact_and_touches_nothing_else(kind, dtype, lens, rows, Hk, d, page):
    c, desc, K, V, cache, dev, starts = write_case(kind, dtype, lens, rows, Hk, d, page, 3, gap=8)
    keys, values, ks, vs = raw_views(desc, cache.cpu().numpy())
    mine = np.zeros((desc.n_pages, page), bool)
    t = 0
    for b, n in enumerate(rows):
        (kc, kstep), (vc, vstep) = (as_codes(x[t:t + n].float().cpu().numpy(), c.int8) for x in (K, V))
        for i in range(n):
            pos = lens[b] - n + i
            p, s = c.table[b, pos // page], pos % page
            mine[p, s] = True
            assert np.array_equal(keys[p, :, s, :d], kc[i]) and not keys[p, :, s, d:].any()
            assert np.array_equal(values[p, :, s // 16, :d, s % 16], vc[i])
            if c.int8:
                assert np.array_equal(ks[p, :, s], kstep[i]) and np.array_equal(vs[p, :, s], vstep[i])
        t += n
    untouched = lambda x: np.array_equal(x, np.full_like(x, -1 if x.dtype == np.int8 else np.iinfo(x.dtype).max))
    assert untouched(keys.transpose(0, 2, 1, 3)[~mine])
    assert untouched(values[..., :d, :].transpose(0, 2, 4, 1, 3).reshape(desc.n_pages, page, -1)[~mine])
    if c.int8:
        assert untouched(ks.transpose(0, 2, 1)[~mine]) and untouched(vs.transpose(0, 2, 1)[~mine])


@pytest.mark.parametrize("kind,out", [(I8, torch.bfloat16), (I8, torch.float32), (BF, torch.bfloat16), (BF, torch.float32)])
@pytest.mark.parametrize("lens,rows,Hk,d,page", SHAPES)
def test_read_gives_what_the_cache_stands_for(kind, out, lens, rows, Hk, d, page):
    """Written in one type, read in another into rows with gaps between; other numbers of rows than were written."""
    c, desc, K, V, cache, dev, starts = write_case(kind, torch.float32, lens, rows, Hk, d, page, 5)
    less = [max(0, n - 2) if n > 4 else n for n in rows]
    T = sum(less)
    bufs = [torch.full((T + 3, Hk * d + 6), 7.0, dtype=out, device="cuda") for _ in range(2)]
    Kr, Vr = (x[:, :Hk * d].unflatten(1, (Hk, d)) for x in bufs)
    pq.kv_read(desc, cache, *dev, Kr, Vr, row_start=torch.tensor(np.concatenate([[0], np.cumsum(less)]), dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    for x, got, buf in ((K, Kr, bufs[0]), (V, Vr, bufs[1])):
        t = s = 0
        for n, m in zip(rows, less):
            want = torch.from_numpy(ao.stored(x[t + n - m:t + n].float().cpu().numpy(), c.int8)).to(out)
            assert torch.equal(got[s:s + m].cpu(), want)
            t, s = t + n, s + m
        assert (buf[T:] == 7).all() and (buf[:, Hk * d:] == 7).all()      # rows behind the last sequence, gaps between the rows


def test_one_row_per_sequence_and_one_of_the_two_outputs():
    c, desc, K, V, cache, dev, _ = write_case(I8, torch.bfloat16, [5, 40, 16], [1, 1, 1], 2, 64, 16, 8)
    again = cache.clone().fill_(255)
    pq.kv_write(desc, K, V, again, *dev)                       # row b is the last token of sequence b
    assert torch.equal(again, cache)
    out = torch.full((4, 2, 64), 7.0, dtype=torch.float32, device="cuda")
    pq.kv_read(desc, cache, *dev, None, out)
    torch.cuda.synchronize()
    assert torch.equal(out[:3].cpu(), torch.from_numpy(ao.stored(V.float().cpu().numpy(), True))) and (out[3] == 7).all()


@pytest.mark.parametrize("kind", [I8, BF])
def test_absent_pages_and_positions(kind):
    """Tokens without a page, before position 0 or beyond the table are dropped and read back as zeros; nothing else is written."""
    page, Hk, d = 16, 2, 64
    c = Paged(kind, [40, 10, 64], Hk, d, page, 4)
    c.table[0, 1] = -5                                         # tokens 16..31 of sequence 0
    c.table[2, 3] = c.n_pages                                  # tokens 48..63 of sequence 2
    lens, rows = [40, 10, 200], [40, 14, 180]                  # 4 rows before position 0; positions beyond max_pages * page
    desc = c.desc()
    cap = desc.max_pages * page
    rng = np.random.default_rng(0)
    K, V = (torch.from_numpy(rng.standard_normal((sum(rows), Hk, d)).astype(np.float32)).cuda() for _ in range(2))
    cache = pq.kv_cache(desc)
    cache.fill_(255)
    t32 = lambda a: torch.tensor(a, dtype=torch.int32).cuda()
    dev, starts = (t32(lens), torch.from_numpy(c.table).cuda()), t32(np.concatenate([[0], np.cumsum(rows)]))
    pq.kv_write(desc, K, V, cache, *dev, row_start=starts)
    Kr, Vr = (torch.full_like(K, 7.0) for _ in range(2))
    pq.kv_read(desc, cache, *dev, Kr, Vr, row_start=starts)
    torch.cuda.synchronize()
    present, t = [], 0
    for b, n in enumerate(rows):
        for i in range(n):
            pos = lens[b] - n + i
            present.append(0 <= pos < cap and 0 <= c.table[b, pos // page] < c.n_pages)
    present = np.array(present)
    assert 0 < present.sum() < len(present)
    for x, got in ((K, Kr), (V, Vr)):
        want = ao.stored(x.cpu().numpy(), c.int8)
        want[~present] = 0
        assert np.array_equal(got.cpu().numpy(), want)
    keys = raw_views(desc, cache.cpu().numpy())[0]
    written = (keys.view(np.uint8) != 255).reshape(desc.n_pages, Hk, page, -1).any(-1).any(1).sum()
    assert written == present.sum()


def test_rows_out_of_order_or_range_stay_inside():
    """row_start that decreases or points outside is wrong, but no access leaves the buffers and foreign rows stay."""
    c = Paged(I8, [32, 32, 32], 2, 64, 16, 4)
    desc = c.desc()
    cache, lens, table = c.device()
    K = torch.randn(20, 2, 64, device="cuda")
    for bad in ([-7, 5, 3, 40], [0, 30, 10, 20], [50, 60, 70, 80], [3, 3, 3, 3]):
        rs = torch.tensor(bad, dtype=torch.int32).cuda()
        pq.kv_write(desc, K, K, cache, lens, table, row_start=rs)
        out = torch.full_like(K, 7.0)
        pq.kv_read(desc, cache, lens, table, out, None, row_start=rs)
        torch.cuda.synchronize()
        assert torch.isfinite(out).all()
    assert (out == 7).all()                                    # every sequence empty: no row is anybody's


def test_rows_that_are_not_finite():
    c, desc, K, V, cache, dev, starts = write_case(I8, torch.float32, [20], [20], 2, 64, 16, 2)
    K[3, 1, 7], K[4, 0, 0], V[5, 1, 63] = float("inf"), float("nan"), float("-inf")
    K[6], V[7] = 0.0, 1e-30
    pq.kv_write(desc, K, V, cache, *dev, row_start=starts)
    Kr, Vr = torch.empty_like(K), torch.empty_like(V)
    pq.kv_read(desc, cache, *dev, Kr, Vr, row_start=starts)
    torch.cuda.synchronize()
    for x, got in ((K, Kr), (V, Vr)):
        want = ao.stored(x.cpu().numpy(), True)
        assert np.array_equal(got.cpu().numpy(), want, equal_nan=True)
    assert torch.isnan(Kr[3, 1]).all() and torch.isnan(Kr[4, 0]).all() and torch.isnan(Vr[5, 1]).all() and torch.isnan(Kr).sum() == 128
    assert (Kr[6] == 0).all()


@pytest.mark.parametrize("kind", [I8, BF])
def test_a_cache_beyond_4_gib(kind):
    """Pages whose offsets pass 32 bits: the last page of a pool of 4.5 GiB."""
    Hk, d, page = 8, 128, 1024
    per_page = pq.lib().pq_kv_cache_bytes(pq.C.byref(pq.make_kv_desc(kind, Hk, d, page, 1, 1, 1)))
    n_pages = int(4.5 * 2 ** 30) // per_page
    desc = pq.make_kv_desc(kind, Hk, d, page, n_pages, 2, 1)
    cache = pq.kv_cache(desc)
    t32 = lambda a: torch.tensor(a, dtype=torch.int32).cuda()
    lens, table = t32([1024, 9]), t32([[n_pages - 1], [3]])
    K, V = (torch.randn(1033, Hk, d, device="cuda") for _ in range(2))
    starts = t32([0, 1024, 1033])
    pq.kv_write(desc, K, V, cache, lens, table, row_start=starts)
    Kr, Vr = torch.empty_like(K), torch.empty_like(V)
    pq.kv_read(desc, cache, lens, table, Kr, Vr, row_start=starts)
    adesc = pq.make_attn_desc(desc, 16)
    Q = torch.randn(2, 16, d, device="cuda").bfloat16()
    O, O2 = torch.empty_like(Q), torch.empty_like(Q)
    pq.attn_decode(adesc, Q, cache, lens, table, O, pq.attn_decode_workspace(adesc))
    pq.attn_prefill(adesc, Q, cache, lens, table, t32([0, 1, 2]), O2)
    torch.cuda.synchronize()
    for x, got in ((K, Kr), (V, Vr)):
        assert np.array_equal(got.cpu().numpy(), ao.stored(x.cpu().numpy(), kind == I8))
    k, v = Kr[:1024, 0].double(), Vr[:1024, 0].double()
    want = torch.softmax(Q[0, :2].double() @ k.t().contiguous() / d ** 0.5, -1) @ v
    for o in (O, O2):
        assert (o[0, :2].double() - want).abs().max() <= 2.0 ** -6 * v.abs().max()
