"""Attention over the rows of a call and its gradients against the definition in fp64."""
import numpy as np
import pytest
import torch

from self_attention_cases import Packed, U
from paper_2602_22592_amd import binding as pq

pytestmark = pytest.mark.gpu

CASES = {
    "one_row": dict(rows=[1], H=1, Hk=1, d=64),
    "one_row_whole": dict(rows=[1, 1, 1], H=2, Hk=1, d=32, causal=False),
    "two_rows": dict(rows=[2], H=4, Hk=2, d=128),
    "d2": dict(rows=[5, 40], H=2, Hk=1, d=2),
    "d6": dict(rows=[70], H=3, Hk=3, d=6),
    "d32": dict(rows=[33, 65], H=4, Hk=4, d=32),
    "d64": dict(rows=[130, 64, 1, 63], H=4, Hk=2, d=64),
    "d80": dict(rows=[129, 31], H=5, Hk=1, d=80),
    "d90": dict(rows=[65, 150], H=2, Hk=2, d=90),
    "d96": dict(rows=[128], H=4, Hk=1, d=96),
    "d98": dict(rows=[100], H=2, Hk=1, d=98),
    "d126": dict(rows=[70, 70], H=2, Hk=2, d=126),
    "d128": dict(rows=[257, 5], H=8, Hk=2, d=128),
    "whole": dict(rows=[200, 33], H=4, Hk=2, d=64, causal=False),
    "whole128": dict(rows=[129], H=2, Hk=2, d=128, causal=False),
    "window1": dict(rows=[140], H=2, Hk=1, d=64, window=1),
    "window2": dict(rows=[70], H=2, Hk=1, d=64, window=2),
    "window100": dict(rows=[400, 50], H=2, Hk=1, d=128, window=100),
    "window64": dict(rows=[300], H=2, Hk=2, d=90, window=64),
    "window_far": dict(rows=[150], H=2, Hk=1, d=64, window=2 ** 31 - 1),
    "empty_between": dict(rows=[0, 70, 0, 0, 3, 0], H=2, Hk=2, d=64),
    "strided": dict(rows=[130, 20], H=4, Hk=2, d=64, gap=16),
    "strided_odd": dict(rows=[130, 20], H=4, Hk=2, d=128, gap=6),
    "others": dict(rows=[66, 7], H=2, Hk=1, d=64, before=3, behind=200),
    "negative_scale": dict(rows=[90], H=2, Hk=1, d=64, scale=-0.1),
    "zero_scale": dict(rows=[90], H=2, Hk=1, d=64, scale=0.0),
    "sharp": dict(rows=[300], H=2, Hk=1, d=128, size=3.0),
    "group16": dict(rows=[100], H=16, Hk=1, d=64),
    "many": dict(rows=[1 + i % 5 for i in range(100)], H=2, Hk=2, d=64),
    # (few tiles of tokens and many stages each: their work is cut and joined)
    "pieces": dict(rows=[300, 5, 400], H=16, Hk=1, d=90, window=100, before=2, behind=3),
    "pieces_whole": dict(rows=[330, 70], H=8, Hk=1, d=32, causal=False),
    "pieces_128": dict(rows=[1, 700], H=8, Hk=2, d=128, scale=-0.05),
    "long": dict(rows=[1500], H=2, Hk=1, d=128, seed=3),
}


@pytest.mark.parametrize("name", CASES)
def test_against_the_definition(name):
    c = Packed(**CASES[name])
    dev = c.inputs()
    O, lse = c.forward(dev)
    c.check_forward(O, lse)
    out = c.backward(O, lse, dev)
    c.check_backward(O, lse, out)
    again = c.backward(O, lse, dev)
    assert all(torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16)) for a, b in zip(out, again))   # (whatever the order of workgroups)


@pytest.mark.parametrize("case", [dict(rows=[1, 2, 17, 64, 3], H=4, Hk=2, d=64), dict(rows=[50, 64], H=8, Hk=1, d=128), dict(rows=[5, 33], H=3, Hk=3, d=90),
                                  dict(rows=[64, 2], H=2, Hk=2, d=32, causal=False), dict(rows=[60, 9], H=4, Hk=4, d=96, window=7)],
                         ids=["grouped", "one_head", "odd", "whole", "window"])
def test_short_sequences_have_the_outputs_rounding_alone(case):
    """Rows that see at most 64 tokens: p and dS are two bf16 numbers each."""
    c = Packed(**case)
    O, lse = c.forward()
    c.check_backward(O, lse, c.backward(O, lse), operand=U * U)


@pytest.mark.parametrize("pieces", [0, 1, 2, 3])
def test_a_workspace_with_room_for_fewer_pieces(pieces):
    c = Packed(rows=[330, 70], H=8, Hk=1, d=64)
    O, lse = c.forward()
    c.check_backward(O, lse, c.backward(O, lse, pieces=pieces))
