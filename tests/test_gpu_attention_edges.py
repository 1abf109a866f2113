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
