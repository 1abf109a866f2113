"""Attention over the rows of a call: what a tile's last rows and other sequences must not change."""
import pytest
import torch

from self_attention_cases import Packed

pytestmark = pytest.mark.gpu


def differing_rows(a, b):
    bits = lambda x: x.contiguous().view(torch.int16 if x.dtype is torch.bfloat16 else torch.int32)
    return (bits(a) != bits(b)).view(len(a), -1).any(1).nonzero().flatten().tolist()


@pytest.mark.parametrize("d", [64, 128, 90])
@pytest.mark.parametrize("rows,window", [(1000, 512), (810, 300), (417, 160), (1023, 256)])
def test_rows_behind_a_causal_sequence_change_nothing(rows, window, d):
    """A sequence that ends inside a tile, and the same one with rows behind it up to the tile's end: no row sees those behind it, so that the shared
    ones come out bit by bit alike.  (The places of the tile behind the last row see no token of the last row's first stages.)"""
    whole = -(-rows // 128) * 128
    long = Packed(rows=[whole], H=2, Hk=1, d=d, window=window)
    short = Packed(rows=[rows], H=2, Hk=1, d=d, window=window)
    short.q, short.k, short.v, short.do = (x[:rows] for x in (long.q, long.k, long.v, long.do))
    (O, lse), (Os, lses) = long.forward(), short.forward()
    short.check_forward(Os, lses)
    assert not differing_rows(O[:rows], Os) and not differing_rows(lse[:rows], lses)
