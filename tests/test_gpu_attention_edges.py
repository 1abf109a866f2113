"""Attention over the cache at the ends of its ranges: the largest windows and lengths, infinities that rows see, many sequences."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from paged_cases import Paged, check, expected
from paper_2602_22592_amd import binding as pq
from test_gpu_attention import BF, I8, queries, rows_of_call, run_decode, run_prefill, t32  # noqa: F401  (rows_of_call: fixture)
from test_gpu_kv_cache import as_codes, raw_views

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 1


@pytest.mark.parametrize("kind", [I8, BF])
@pytest.mark.parametrize("window", [MOST, MOST - 20, 2 ** 30])
@pytest.mark.usefixtures("rows_of_call")
def test_the_largest_windows_hide_nothing(kind, window):
    """More rows than tokens (positions below 0) under a window that no sequence fills: the rows of a call without one, in few and in many rows."""
    c = Paged(kind, [20, 150, 3], 1, 64, 16, 3)
    rows = [30, 150, 70]
    keep = np.r_[10:180, 247:250]
    Q, q = queries(sum(rows), 2, 64, 6)
    dev = c.device()
    plain = run_prefill(c, Q, rows, 2, dev=dev)
    O, lse = run_prefill(c, Q, rows, 2, window=window, dev=dev)
    assert torch.equal(O, plain[0]) and torch.equal(lse, plain[1])
    check(O[keep], lse[keep], expected(c, q[keep], [20, 150, 3], 0.125, p_bits=8), f"window {window}")
    hidden = np.setdiff1d(np.arange(sum(rows)), keep)
    assert (O[hidden] == 0).all() and torch.isneginf(lse[hidden]).all()
    plain = run_decode(c, Q[:3], 2, dev=dev)
    one = run_decode(c, Q[:3], 2, window=window, dev=dev)
    assert torch.equal(one[0], plain[0]) and torch.equal(one[1], plain[1])


@pytest.mark.parametrize("kind", [I8, BF])
@pytest.mark.usefixtures("rows_of_call")
def test_lengths_far_beyond_the_table(kind):
    """Lengths up to 2^31 - 1: a row whose window lies behind what the table holds sees nothing, one without a window sees what it holds."""
    c = Paged(kind, [64, 40, 33], 1, 64, 16, 3)
    cache, _, table = c.device()
    Q, q = queries(3, 2, 64, 6)
    lens = t32([MOST, 40, MOST - 64])
    O, lse = run_decode(c, Q, 2, window=40, dev=(cache, lens, table))
    want = expected(c, q, [1, 1, 1], 0.125, window=40, p_bits=15, fixed_point=kind == I8)
    check(O[1:2], lse[1:2], tuple(x[1:2] for x in want), "within the table")
    assert (O[::2] == 0).all() and torch.isneginf(lse[::2]).all()
    want = expected(c, q, [1, 1, 1], 0.125, p_bits=15, fixed_point=kind == I8)
    check(*run_decode(c, Q, 2, dev=(cache, t32([MOST, 40, 33]), table)), want, "no window")
    O, lse = run_prefill(c, Q, [1, 1, 1], 2, window=40, dev=(cache, lens, table))
    want = expected(c, q, [1, 1, 1], 0.125, window=40, p_bits=8)
    check(O[1:2], lse[1:2], tuple(x[1:2] for x in want), "a prompt within the table")
    assert (O[::2] == 0).all() and torch.isneginf(lse[::2]).all()


SEEN = [  # token, element, value: elements 3 and 9 hold both infinities, for the rows that see both tokens
    (3, 0, np.inf), (70, 1, -np.inf), (70, 2, np.nan), (95, 9, -np.inf), (128, 9, np.inf), (139, 3, np.inf), (150, 3, -np.inf), (150, 63, np.inf),
    (180, 33, -np.inf), (199, 40, np.inf),
]
WEIGHTS = {"ordinary": None, "one": 400.0, "none": -2400.0}    # the first element of those tokens' keys, at a query of 1 and a scale of 1/8


def with_infinities(kind, L, weight, Hk=1, d=64, page=16, shift=0):
    """A sequence with SEEN in the first key-value head's values; "one": their tokens' weight is 1 together, "none": below e^-290, which fp32
    does not hold (the definition in fp64 does)."""
    c = Paged(kind, [L], Hk, d, page, 5)
    if WEIGHTS[weight] is not None:
        c.K[0][:, 0, 0] = 0.0
    for t, e, x in SEEN:
        c.V[0][t + shift, 0, e] = x
        if WEIGHTS[weight] is not None:
            c.K[0][t + shift, 0, 0] = WEIGHTS[weight]
    return c


def check_nonfinite(O, lse, ref, name):
    """Infinities and NaN where the definition has them, the other elements within their bounds."""
    o, l, tol, tl = ref
    got = O.float().cpu().numpy()
    for f in (np.isnan, np.isposinf, np.isneginf):
        assert np.array_equal(f(got), f(o)), (name, f.__name__, np.argwhere(f(got) != f(o))[:5])
    fin = np.isfinite(o)
    assert 0 < fin.sum() < fin.size or np.isnan(o).any(), name
    assert (np.abs(got - o)[fin] <= tol[fin]).all(), name
    assert (np.abs(lse.cpu().numpy() - l) <= tl).all(), name


@pytest.mark.filterwarnings("ignore::RuntimeWarning")
@pytest.mark.parametrize("kind", [I8, BF])
@pytest.mark.parametrize("weight", list(WEIGHTS))
@pytest.mark.parametrize("L,shift,d,window", [(200, 0, 64, 0), (200, 0, 64, 90), (203, 0, 90, 0), (2600, 2300, 64, 0), (4500, 100, 64, 0), (200, 0, 160, 0)])
def test_decode_infinities_that_are_seen(kind, weight, L, shift, d, window):
    """Whole sequences and pieces, whatever the tokens weigh."""
    c = with_infinities(kind, L, weight, Hk=2, d=d, shift=shift)
    Q, q = queries(1, 6, d, 6)
    Q[..., 0], q[..., 0] = 1.0, 1.0
    O, lse = run_decode(c, Q, 6, window=window, scale=0.125)
    check_nonfinite(O, lse, expected(c, q, [1], 0.125, window=window, p_bits=15, fixed_point=kind == I8), f"{weight} {L}")


@pytest.mark.filterwarnings("ignore::RuntimeWarning")
@pytest.mark.parametrize("kind", [I8, BF])
@pytest.mark.parametrize("weight", list(WEIGHTS))
@pytest.mark.parametrize("rows,G,d,causal,window", [(200, 1, 64, True, 0), (61, 3, 64, True, 0), (200, 2, 64, True, 50), (40, 2, 90, False, 0), (70, 1, 160, True, 100), (70, 1, 192, True, 100)])
@pytest.mark.usefixtures("rows_of_call")
def test_prompt_infinities_that_are_seen(kind, weight, rows, G, d, causal, window):
    """In tiles that all rows see and in those that some rows see a part of."""
    c = with_infinities(kind, 200, weight, Hk=2, d=d)
    Q, q = queries(rows, 2 * G, d, 6)
    Q[..., 0], q[..., 0] = 1.0, 1.0
    O, lse = run_prefill(c, Q, [rows], 2 * G, causal=causal, window=window, scale=0.125)
    check_nonfinite(O, lse, expected(c, q, [rows], 0.125, causal=causal, window=window, p_bits=8), weight)


@pytest.mark.parametrize("kind", [I8, BF])
@pytest.mark.usefixtures("rows_of_call")
def test_rows_all_of_whose_scores_are_minus_infinity_are_nan(kind):
    """.. whatever the values are, infinities among them; the head beside it is not touched."""
    c = Paged(kind, [150], 2, 64, 16, 5)
    clean = Paged(kind, [150], 2, 64, 16, 5)
    c.K[0][:, 0, 0] = -np.inf
    c.V[0][::9, 0, 7], c.V[0][::13, 0, 11] = np.inf, -np.inf
    Q, _ = queries(150, 2, 64, 6)
    Q[..., 0] = 1.0
    for run, n in ((run_prefill, 150), (run_decode, 1)):
        args = ([150],) if run is run_prefill else ()
        O, lse = run(c, Q[150 - n:], *args, 2)
        want = run(clean, Q[150 - n:], *args, 2)
        assert torch.isnan(O[:, 0].float()).all() and torch.equal(O[:, 1], want[0][:, 1]) and torch.equal(lse[:, 1], want[1][:, 1])


def many_sequences(B, kind, seed, longest=9):
    """Ragged sequences, every third without rows, many of one token; rows are the last ones of their sequences."""
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, longest + 1, B)
    lens[rng.random(B) < 0.3] = 1
    rows = np.minimum(lens, rng.integers(0, longest + 1, B))
    rows[::3] = 0
    lens[-1] = rows[-1] = longest
    return Paged(kind, lens.tolist(), 2, 32, 16, seed), lens, rows


SEARCHES = [64, 65, 130, 1000, 4097, 4200]                     # sequences: one, two and three steps of 64 entries


@pytest.mark.parametrize("kind", [I8, BF])
@pytest.mark.parametrize("B", SEARCHES)
@pytest.mark.parametrize("before", [0, 5])
def test_cache_calls_of_many_sequences(kind, B, before):
    """Every row lies where its sequence's table says, nothing else is written, and it reads back; rows before the first sequence's are nobody's."""
    c, lens, rows = many_sequences(B, kind, B)
    desc = c.desc()
    T, page = int(rows.sum()), c.page
    starts = np.concatenate([[0], np.cumsum(rows)]) + before
    rng = np.random.default_rng(1)
    K, V = (torch.from_numpy(rng.standard_normal((before + T + 4, 2, 32)).astype(np.float32)).cuda() for _ in range(2))
    cache = pq.kv_cache(desc)
    cache.fill_(255)
    dev, rs = (t32(lens), torch.from_numpy(c.table).cuda()), t32(starts)
    pq.kv_write(desc, K, V, cache, *dev, row_start=rs)
    outs = [torch.full_like(K, 7.0) for _ in range(2)]
    pq.kv_read(desc, cache, *dev, *outs, row_start=rs)
    torch.cuda.synchronize()
    seq = np.repeat(np.arange(B), rows)
    pos = lens[seq] - rows[seq] + np.arange(T) - (starts[seq] - before)
    at, slot = c.table[seq, pos // page], pos % page
    keys, values, ks, vs = raw_views(desc, cache.cpu().numpy())
    own = slice(before, before + T)
    (kc, kstep), (vc, vstep) = (as_codes(x[own].cpu().numpy(), c.int8) for x in (K, V))
    assert np.array_equal(keys[at, :, slot], kc) and np.array_equal(values[at, :, slot // 16, :, slot % 16], vc)
    if c.int8:
        assert np.array_equal(ks[at, :, slot], kstep) and np.array_equal(vs[at, :, slot], vstep)
    mine = np.zeros((c.n_pages, page), bool)
    mine[at, slot] = True
    assert mine.sum() == T                                     # (every row has a place of its own)
    assert (keys.view(np.uint8).reshape(c.n_pages, 2, page, -1).transpose(0, 2, 1, 3)[~mine] == 255).all()
    assert (np.ascontiguousarray(values.transpose(0, 2, 4, 1, 3)).view(np.uint8).reshape(c.n_pages, page, -1)[~mine] == 255).all()
    for x, got in zip((K, V), outs):
        assert np.array_equal(got[own].cpu().numpy(), ao.stored(x[own].cpu().numpy(), c.int8))
        assert (got[:before] == 7).all() and (got[before + T:] == 7).all()


@pytest.mark.parametrize("kind", [I8, BF])
@pytest.mark.parametrize("B", SEARCHES)
@pytest.mark.parametrize("before", [0, 5])
@pytest.mark.parametrize("many", [False, True])
def test_prompts_of_many_sequences(kind, B, before, many):
    """.. in few rows (32 a tile) and in many (128 a tile)."""
    c, lens, rows = many_sequences(B, kind, B + 1)
    cache, dlens, table = c.device()
    T, H = int(rows.sum()), 4 if many else 2
    total = max(before + T + 2, 16384 // H + 1 if many else 0)
    assert many == (total * H > 16384)
    Q, q = queries(total, H, 32, 6)
    O, lse = torch.full((total, H, 32), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((total, H), 7.0, device="cuda")
    pq.attn_prefill(pq.make_attn_desc(c.desc(), H), Q, cache, dlens, table, t32(np.concatenate([[0], np.cumsum(rows)]) + before), O, lse=lse)
    torch.cuda.synchronize()
    own = slice(before, before + T)
    check(O[own], lse[own], expected(c, q[own], rows.tolist(), 32 ** -0.5, p_bits=8), f"{B} sequences, {T} rows")
    for x in (O, lse):
        assert (x[:before] == 7).all() and (x[before + T:] == 7).all()


@pytest.mark.parametrize("kind", [I8, BF])
@pytest.mark.parametrize("B,T", [(64, 64), (65, 65), (130, 100), (4100, 4100), (4100, 9)])
def test_last_tokens_of_many_sequences_as_prompts(kind, B, T):
    """No row_start: row b is the last token of sequence b, as many as there are rows."""
    c, lens, _ = many_sequences(B, kind, B + 2)
    cache, dlens, table = c.device()
    Q, q = queries(T, 4, 32, 6)
    O, lse = torch.full((T, 4, 32), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((T, 4), 7.0, device="cuda")
    pq.attn_prefill(pq.make_attn_desc(c.desc(), 4), Q, cache, dlens, table, None, O, lse=lse)
    torch.cuda.synchronize()
    few = Paged.__new__(Paged)
    few.__dict__.update(c.__dict__, B=T)
    check(O, lse, expected(few, q, [1] * T, 32 ** -0.5, p_bits=8), f"{T} of {B}")
