"""Attention over the paged key-value cache against the definition in fp64: one token per sequence, and the rows of prompts."""
import sys

import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from paged_cases import Paged, check, expected
from paper_2602_22592_amd import binding as pq

pytestmark = pytest.mark.gpu
BF, I8 = pq.PQ_KV_BF16, pq.PQ_KV_INT8
t32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32).cuda()


def starts_of(rows):
    return t32(np.concatenate([[0], np.cumsum(rows)]))


def queries(T, H, d, seed, scale=1.0, gap=0):
    """bf16 rows [T][H][d] on the GPU (with `gap` elements between them) and their values."""
    x = ao.bf16(np.random.default_rng(seed).standard_normal((T, H, d)) * scale)
    buf = torch.full((T, H * d + gap), float("nan"), dtype=torch.bfloat16, device="cuda")
    buf[:, :H * d] = torch.from_numpy(x.reshape(T, H * d)).cuda().bfloat16()
    return buf[:, :H * d].unflatten(1, (H, d)), x


def run_decode(c, Q, H, window=0, max_len=0, scale=None, dev=None, lens=None):
    cache, dlens, table = dev or c.device()
    desc = pq.make_attn_desc(c.desc(), H, scale=scale, window=window, max_len=max_len)
    ws = pq.attn_decode_workspace(desc)
    ws.fill_(255)
    O = torch.full((c.B, H, c.d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((c.B, H), float("nan"), device="cuda")
    pq.attn_decode(desc, Q, cache, dlens if lens is None else lens, table, O, ws, lse=lse)
    torch.cuda.synchronize()
    return O, lse


LEAST_ROWS = 0


@pytest.fixture(params=["few", "many"])
def rows_of_call(request, monkeypatch):
    """Prompts alone, and followed by so many rows of no sequence that the call counts as one of many rows (another kernel)."""
    monkeypatch.setattr(sys.modules[__name__], "LEAST_ROWS", 0 if request.param == "few" else 16385)


def run_prefill(c, Q, rows, H, causal=True, window=0, scale=None, dev=None):
    cache, dlens, table = dev or c.device()
    if Q.shape[0] * H < LEAST_ROWS:
        buf = torch.full((-(-LEAST_ROWS // H), Q.stride(0)), float("nan"), dtype=torch.bfloat16, device="cuda")
        buf[:Q.shape[0], :H * c.d] = Q.reshape(-1, H * c.d)
        Q = buf[:, :H * c.d].unflatten(1, (H, c.d))
    desc = pq.make_attn_desc(c.desc(), H, scale=scale, causal=causal, window=window)
    O = torch.full((Q.shape[0], H, c.d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((Q.shape[0], H), 7.0, device="cuda")
    pq.attn_prefill(desc, Q, cache, dlens, table, starts_of(rows), O, lse=lse)
    torch.cuda.synchronize()
    T = sum(rows)
    assert (O[T:] == 7).all() and (lse[T:] == 7).all()
    return O[:T], lse[:T]


DECODE = [  # lens, Hk, group, d, page
    ([1], 1, 1, 64, 16), ([0, 1, 15, 16, 17, 63, 64, 65], 2, 1, 64, 16), ([300, 2, 129], 3, 4, 128, 32), ([77, 500], 2, 5, 90, 64),
    ([1000, 31, 0, 257], 1, 8, 64, 128), ([130], 2, 16, 128, 16), ([200, 64], 1, 20, 32, 16), ([95, 700], 2, 2, 256, 64),
    ([33], 4, 3, 2, 16), ([400, 10], 1, 32, 80, 32), ([90, 128], 2, 7, 96, 1024), ([70, 190], 1, 6, 160, 16), ([333], 2, 9, 224, 32),
    ([65, 0, 300, 1, 129, 64, 63, 200] * 6, 6, 1, 64, 16), ([65, 0, 300, 1, 129] * 6, 9, 3, 90, 32), ([128, 5, 77] * 10, 9, 1, 128, 16), ([9, 70] * 15, 9, 5, 32, 16),
]


@pytest.mark.parametrize("kind", [I8, BF])
@pytest.mark.parametrize("lens,Hk,G,d,page", DECODE)
def test_decode(kind, lens, Hk, G, d, page):
    c = Paged(kind, lens, Hk, d, page, 11)
    Q, q = queries(c.B, Hk * G, d, 5, gap=8 if d % 8 == 0 else 2)
    O, lse = run_decode(c, Q, Hk * G)
    check(O, lse, expected(c, q, [1] * c.B, d ** -0.5, p_bits=15, fixed_point=kind == I8), "decode")


@pytest.mark.parametrize("kind", [I8, BF])
@pytest.mark.parametrize("max_len", [1, 300, 1300, 5000])
def test_decode_long_and_any_bound(kind, max_len):
    """Long histories, cut into pieces by a bound that may be smaller than they are; the same numbers whatever the cut."""
    c = Paged(kind, [5000, 1, 0, 1299, 64], 2, 64, 64, 3)
    Q, q = queries(c.B, 8, 64, 6)
    O, lse = run_decode(c, Q, 8, max_len=max_len)
    check(O, lse, expected(c, q, [1] * c.B, 0.125, p_bits=15, fixed_point=kind == I8), f"max_len {max_len}")
    O2, lse2 = run_decode(c, Q, 8, max_len=max_len)
    assert torch.equal(O, O2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("kind", [I8, BF])
@pytest.mark.parametrize("window", [1, 16, 63, 64, 100, 1000])
def test_decode_window(kind, window):
    c = Paged(kind, [500, 64, 1, 65, 101], 2, 64, 16, 3)
    Q, q = queries(c.B, 4, 64, 6)
    O, lse = run_decode(c, Q, 4, window=window, max_len=500)
    check(O, lse, expected(c, q, [1] * c.B, 0.125, window=window, p_bits=15, fixed_point=kind == I8), f"window {window}")


@pytest.mark.parametrize("kind", [I8, BF])
def test_decode_sharp_flat_and_negative_scores(kind):
    """Scores of hundreds (one token takes all), a scale of zero (the mean), a negative scale, queries far from 1."""
    c = Paged(kind, [700, 40], 2, 64, 32, 9, key_scale=4.0)
    for scale, mul in ((3.0, 4.0), (0.0, 1.0), (-0.125, 1.0), (0.125, 2.0 ** -60), (2.0 ** -70, 2.0 ** 70)):
        Q, q = queries(c.B, 4, 64, 6, scale=mul)
        O, lse = run_decode(c, Q, 4, scale=scale)
        check(O, lse, expected(c, q, [1, 1], np.float32(scale), p_bits=15, fixed_point=kind == I8), f"scale {scale} queries {mul}")


@pytest.mark.parametrize("kind", [I8, BF])
def test_decode_values_of_very_different_size(kind):
    """Values a million times larger at tokens that hardly count, and at the one that does."""
    c = Paged(kind, [300], 1, 64, 16, 9, key_scale=3.0)
    c.V[0][::7] *= 2.0 ** 20
    c.V[0][5::11] *= 2.0 ** -20
    Q, q = queries(1, 2, 64, 6, scale=2.0)
    O, lse = run_decode(c, Q, 2)
    check(O, lse, expected(c, q, [1], 0.125, p_bits=15, fixed_point=kind == I8), "values")


PREFILL = [  # lens, rows, Hk, group, d, page
    ([1], [1], 1, 1, 64, 16), ([5, 0, 17, 40], [5, 0, 17, 40], 2, 1, 64, 16), ([130], [130], 1, 2, 128, 32), ([300, 64], [70, 1], 2, 4, 90, 64),
    ([257, 128, 33], [257, 128, 2], 1, 3, 64, 128), ([150], [150], 1, 5, 256, 16), ([96, 31], [96, 31], 2, 1, 32, 16), ([66], [65], 1, 8, 80, 32),
    ([200], [3], 2, 2, 96, 1024), ([65, 64, 63], [65, 64, 63], 1, 1, 2, 16), ([70], [70], 1, 2, 160, 16), ([140], [139], 1, 1, 224, 64),
    ([90], [90], 1, 2, 192, 32), ([9, 70, 0, 33, 1, 64, 128, 5, 0, 31, 90, 200], [9, 60, 0, 33, 1, 64, 100, 2, 0, 31, 90, 33], 2, 2, 64, 16),
]


@pytest.mark.parametrize("kind", [I8, BF])
@pytest.mark.parametrize("lens,rows,Hk,G,d,page", PREFILL)
@pytest.mark.usefixtures("rows_of_call")
def test_prefill(kind, lens, rows, Hk, G, d, page):
    c = Paged(kind, lens, Hk, d, page, 12)
    Q, q = queries(sum(rows) + 3, Hk * G, d, 5, gap=8 if d % 8 == 0 else 2)
    O, lse = run_prefill(c, Q, rows, Hk * G)
    check(O, lse, expected(c, q, rows, d ** -0.5, p_bits=8), "prefill")


@pytest.mark.parametrize("kind", [I8, BF])
@pytest.mark.parametrize("causal,window", [(False, 0), (True, 1), (True, 17), (True, 64), (True, 150)])
@pytest.mark.usefixtures("rows_of_call")
def test_prefill_masks(kind, causal, window):
    c = Paged(kind, [260, 64, 100], 2, 64, 16, 3)
    rows = [200, 64, 1]
    Q, q = queries(sum(rows), 4, 64, 6)
    O, lse = run_prefill(c, Q, rows, 4, causal=causal, window=window)
    check(O, lse, expected(c, q, rows, 0.125, causal=causal, window=window, p_bits=8), f"causal {causal} window {window}")


@pytest.mark.parametrize("kind", [I8, BF])
@pytest.mark.usefixtures("rows_of_call")
def test_prefill_sharp_flat_and_negative_scores(kind):
    c = Paged(kind, [150], 2, 64, 32, 9, key_scale=4.0)
    for scale, mul in ((3.0, 4.0), (0.0, 1.0), (-0.125, 1.0), (2.0 ** -70, 2.0 ** 70)):
        Q, q = queries(150, 4, 64, 6, scale=mul)
        O, lse = run_prefill(c, Q, [150], 4, scale=scale)
        check(O, lse, expected(c, q, [150], np.float32(scale), p_bits=8), f"scale {scale} queries {mul}")


@pytest.mark.parametrize("kind", [I8, BF])
@pytest.mark.usefixtures("rows_of_call")
def test_absent_pages_are_attended_by_nobody(kind):
    """Pages without an entry in the middle and at the end of sequences; one sequence without any page; a row before position 0."""
    c = Paged(kind, [200, 70, 40], 2, 64, 16, 3)
    dev = c.device()
    table = c.table.copy()
    table[0, 2], table[0, 5], table[0, 12], table[1, :], table[2, 0] = -1, c.n_pages + 7, -100, -1, 2 ** 31 - 1
    dev = (dev[0], dev[1], torch.from_numpy(table).cuda())
    present = [np.repeat([0 <= p < c.n_pages for p in table[b]], 16)[:n] for b, n in enumerate(c.lens)]
    Q, q = queries(3, 8, 64, 6)
    check(*run_decode(c, Q, 8, dev=dev), expected(c, q, [1, 1, 1], 0.125, present=present, p_bits=15, fixed_point=kind == I8), "decode")
    rows = [150, 70, 40]
    Q, q = queries(sum(rows), 2, 64, 6)
    check(*run_prefill(c, Q, rows, 2, dev=dev), expected(c, q, rows, 0.125, present=present, p_bits=8), "prefill")


@pytest.mark.parametrize("kind", [I8, BF])
@pytest.mark.usefixtures("rows_of_call")
def test_rows_before_the_first_position_and_beyond_the_table(kind):
    """More rows than tokens: the first see nothing.  More tokens than the table holds: those that it holds are attended."""
    c = Paged(kind, [20, 64], 1, 64, 16, 3)
    cache, lens, table = c.device()
    Q, q = queries(30 + 64, 2, 64, 6)
    O, l = run_prefill(c, Q, [30, 64], 2, dev=(cache, lens, table))
    assert (O[:10] == 0).all() and torch.isneginf(l[:10]).all()
    keep = np.r_[10:30, 30:94]
    check(O[10:], l[10:], expected(c, q[keep], [20, 64], 0.125, p_bits=8), "rows before 0")
    cap = c.max_pages * 16                                     # the last entry of sequence 1's row holds no page
    more = t32([20, cap + 1000])
    Q, q = queries(2, 2, 64, 7)
    O, l = run_decode(c, Q, 2, dev=(cache, more, table))
    check(O, l, expected(c, q, [1, 1], 0.125, p_bits=15, fixed_point=kind == I8), "beyond the table")


@pytest.mark.parametrize("kind", [I8, BF])
@pytest.mark.usefixtures("rows_of_call")
def test_tokens_that_are_not_seen_have_no_effect(kind):
    """Infinities and NaN in keys and values behind a row (causal), before its window and behind the sequence's end."""
    lens, rows, window = [150, 40], [130, 40], 40
    c = Paged(kind, lens, 2, 64, 16, 3)
    Q, q = queries(sum(rows), 4, 64, 6)
    clean = run_prefill(c, Q, rows, 4, window=window)
    clean_one = run_decode(c, Q[:2], 4, window=window)
    bad = {20: float("nan"), 70: float("inf"), 71: float("-inf"), 149: float("nan"), 130: 3e38}
    for t, x in bad.items():
        c.K[0][t, 0, 3] = x
        c.V[0][t, :, 5:60] = x
    O, lse = run_prefill(c, Q, rows, 4, window=window)
    one = run_decode(c, Q[:2], 4, window=window)
    hit = np.zeros(sum(rows), bool)
    for i in range(130):
        hit[i] = any(max(0, 20 + i - window + 1) <= t <= 20 + i for t in bad)
    assert 0 < hit.sum() < 130
    ok = torch.from_numpy(~hit).cuda()
    assert torch.equal(O[ok], clean[0][ok]) and torch.equal(lse[ok], clean[1][ok])
    assert not torch.isfinite(O[:130][torch.from_numpy(hit[:130]).cuda()].float()).all()
    assert torch.equal(one[0][1], clean_one[0][1]) and torch.equal(one[1][1], clean_one[1][1])
    assert torch.isnan(one[0][0, 2:, 5:60].float()).all()      # a NaN that is seen comes out
    c2 = Paged(kind, [110], 2, 64, 16, 3)                      # decode: bad tokens before the window only
    clean_one = run_decode(c2, Q[:1], 4, window=30)
    for t in (5, 79):
        c2.K[0][t], c2.V[0][t] = float("nan"), float("inf")
    one = run_decode(c2, Q[:1], 4, window=30)
    assert torch.equal(one[0], clean_one[0]) and torch.equal(one[1], clean_one[1])


@pytest.mark.parametrize("kind", [I8, BF])
@pytest.mark.usefixtures("rows_of_call")
def test_queries_that_are_not_finite_spoil_their_own_row_alone(kind):
    c = Paged(kind, [90, 40], 2, 64, 16, 3)
    Q, _ = queries(130, 4, 64, 6)
    clean = run_prefill(c, Q, [90, 40], 4)
    clean_one = run_decode(c, Q[:2], 4)
    for r, h, x in ((0, 1, float("inf")), (50, 2, float("nan"))):
        Q[r, h, 7] = x
    O, _ = run_prefill(c, Q, [90, 40], 4)
    one, _ = run_decode(c, Q[:2], 4)
    bad = torch.zeros((130, 4), dtype=torch.bool, device="cuda")
    bad[0, 1] = bad[50, 2] = True
    assert torch.isnan(O[bad].float()).all() and torch.equal(O[~bad], clean[0][~bad])
    assert torch.isnan(one[0, 1].float()).all() and torch.equal(one[~bad[:2]], clean_one[0][~bad[:2]])


@pytest.mark.parametrize("kind", [I8, BF])
def test_a_cache_that_grows_token_by_token(kind):
    """A prompt enters the cache and attends; then tokens are written and attend one at a time.  Every step equals the same row of one
    long prompt (within the two forms' bounds), and a captured step replayed with other contents gives what the eager one gives."""
    B, Hk, G, d, page, n0, steps = 3, 2, 4, 64, 16, 45, 6
    H = Hk * G
    full = [n0 + steps, n0 - 20 + steps, steps]
    c = Paged(kind, full, Hk, d, page, 21)
    desc, adesc = c.desc(), pq.make_attn_desc(c.desc(), H, max_len=max(full))
    cache = pq.kv_cache(desc)
    cache.fill_(255)
    table = torch.from_numpy(c.table).cuda()
    K, V = ([torch.from_numpy(x).cuda().bfloat16() for x in y] for y in (c.K, c.V))
    Q, q = queries(sum(full), H, d, 4)
    at = np.concatenate([[0], np.cumsum(full)])
    first = [n - steps for n in full]
    cat = lambda xs, lo, hi: torch.cat([x[a:b] for x, a, b in zip(xs, lo, hi)])
    pq.kv_write(desc, cat(K, [0] * 3, first), cat(V, [0] * 3, first), cache, t32(first), table, row_start=starts_of(first))
    Qp = torch.cat([Q[a:a + n] for a, n in zip(at, first)])
    Op, lp = torch.empty((sum(first), H, d), dtype=torch.bfloat16, device="cuda"), torch.empty((sum(first), H), device="cuda")
    pq.attn_prefill(adesc, Qp, cache, t32(first), table, starts_of(first), Op, lse=lp)
    ref = expected(c, q, full, d ** -0.5, p_bits=8, fixed_point=kind == I8)
    pick = np.concatenate([np.arange(a, a + n) for a, n in zip(at, first)])
    check(Op, lp, tuple(x[pick] for x in ref), "prompt")
    ws = pq.attn_decode_workspace(adesc)
    k1, v1, q1 = (torch.empty((B, h, d), dtype=torch.bfloat16, device="cuda") for h in (Hk, Hk, H))
    O, lse, lens = torch.empty_like(q1), torch.empty((B, H), device="cuda"), t32(first)

    def step():
        lens.add_(1)
        pq.kv_write(desc, k1, v1, cache, lens, table)
        pq.attn_decode(adesc, q1, cache, lens, table, O, ws, lse=lse)

    graph = None
    for i in range(steps):
        for b in range(B):
            k1[b], v1[b], q1[b] = K[b][first[b] + i], V[b][first[b] + i], Q[at[b] + first[b] + i]
        if i < 2:
            step()
        elif i == 2:
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                step()
            graph.replay()
        else:
            graph.replay()
        torch.cuda.synchronize()
        row = np.array([at[b] + first[b] + i for b in range(B)])
        check(O, lse, tuple(x[row] for x in ref), f"step {i}")


def test_calls_on_other_streams_and_a_fused_projection():
    """Rows that are parts of one fused projection; two streams, a workspace each."""
    Hk, H, d = 2, 8, 64
    c = Paged(I8, [100, 33], Hk, d, 16, 2)
    cache, lens, table = c.device()
    fused = torch.randn(2, (H + 2 * Hk) * d, device="cuda").bfloat16()
    Q = fused[:, :H * d].unflatten(1, (H, d))
    want = run_decode(c, Q.contiguous(), H, dev=(cache, lens, table))
    desc = pq.make_attn_desc(c.desc(), H, max_len=128)
    got = []
    torch.cuda.synchronize()
    for s in (torch.cuda.Stream(), torch.cuda.Stream()):
        with torch.cuda.stream(s):
            ws, O, lse = pq.attn_decode_workspace(desc), torch.empty((2, H, d), dtype=torch.bfloat16, device="cuda"), torch.empty((2, H), device="cuda")
            pq.attn_decode(desc, Q, cache, lens, table, O, ws, lse=lse)
            got.append((O, lse, ws))
    torch.cuda.synchronize()
    for O, lse, _ in got:
        assert torch.equal(O, got[0][0]) and torch.equal(lse, got[0][1])
    assert (got[0][0].float() - want[0].float()).abs().max() <= 2.0 ** -7 * want[0].float().abs().max()


@pytest.mark.usefixtures("rows_of_call")
def test_scores_of_minus_infinity_come_first():
    """64 seen tokens whose scores are -infinity, then scores around -600: the softmax is that of the later ones."""
    c = Paged(BF, [200], 1, 64, 16, 3)
    c.K[0][:, 0, 0], c.K[0][:, 0, 1] = 0.0, -600.0
    c.K[0][:64, 0, 0] = -np.inf
    Q, q = queries(100, 2, 64, 6)
    Q[..., :2], q[..., :2] = 1.0, 1.0
    later = [np.arange(200) >= 64]                             # what counts
    check(*run_prefill(c, Q, [100], 2, scale=1.0), expected(c, q, [100], 1.0, present=later, p_bits=8), "prefill")
    check(*run_decode(c, Q[99:], 2, scale=1.0), expected(c, q[99:], [1], 1.0, present=later, p_bits=15), "decode")


@pytest.mark.parametrize("kind", [I8, BF])
@pytest.mark.parametrize("T", [120, 9000])
def test_a_prompt_captured_and_replayed_with_other_lengths(kind, T):
    """The first call of its kind is a captured one (few rows, many rows); every replay, with other rows, lengths and pages, equals the eager calls."""
    B, Hk, H, d, page, max_pages = 3, 1, 2, 190, 32, 8
    n_pages = B * max_pages
    kv = pq.make_kv_desc(kind, Hk, d, page, n_pages, B, max_pages)
    at = pq.make_attn_desc(kv, H, window=70)
    bf = lambda *s: torch.randn(s, device="cuda").bfloat16()
    K, V, Q = bf(T, Hk, d), bf(T, Hk, d), bf(T, H, d)
    O, lse, K2, V2 = torch.zeros_like(Q), torch.zeros((T, H), device="cuda"), torch.zeros_like(K), torch.zeros_like(V)
    cache, lens, rows = pq.kv_cache(kv), t32([100, 15, 0]), t32([0, 80, 95, 95])
    table = torch.arange(n_pages, dtype=torch.int32, device="cuda").view(B, max_pages).contiguous()
    cache.zero_()

    def calls(cache, O, lse, K2, V2):
        pq.kv_write(kv, K, V, cache, lens, table, row_start=rows)
        pq.attn_prefill(at, Q, cache, lens, table, rows, O, lse=lse)
        pq.kv_read(kv, cache, lens, table, K2, V2, row_start=rows)

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        calls(cache, O, lse, K2, V2)
    for n, r in (([100, 15, 0], [0, 80, 95, 95]), ([0, 256, 33], [0, 0, 87, 120]), ([40, 40, 40], [0, 40, 80, 120]), ([300, 1, 2], [3, 60, 61, 62])):
        lens.copy_(t32(n)), rows.copy_(t32(r))
        table.copy_(torch.randperm(n_pages, device="cuda").int().view(B, max_pages))
        for x in (K, V, Q):
            x.normal_()
        for x in (O, lse, K2, V2):
            x.fill_(7)
        own = [cache.clone(), *(x.clone() for x in (O, lse, K2, V2))]
        torch.cuda.synchronize()
        graph.replay()
        calls(*own)
        torch.cuda.synchronize()
        for x, y in zip((cache, O, lse, K2, V2), own):
            assert torch.equal(x, y)
        for x in (O, lse, K2, V2):                             # rows of no sequence
            assert (x[:r[0]] == 7).all() and (x[r[-1]:] == 7).all()
