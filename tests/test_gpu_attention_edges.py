"""Attention over the cache at the ends of its ranges: the largest windows and lengths, infinities that rows see, many sequences."""
import numpy as np
import pytest
import torch

from paged_cases import Paged, check, expected
from paper_2602_22592_amd import binding as pq
from test_gpu_attention import BF, I8, queries, rows_of_call, run_decode, run_prefill, t32  # noqa: F401  (rows_of_call: fixture)

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
@pytest.mark.parametrize("rows,G,d,causal,window", [(200, 1, 64, True, 0), (61, 3, 64, True, 0), (200, 2, 64, True, 50), (40, 2, 90, False, 0), (70, 1, 160, True, 100)])
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
