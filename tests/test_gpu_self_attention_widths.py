"""Attention over the rows of a call at the widths, alignments and numbers of sequences that choose another kernel, staging or search."""
import pytest
import torch

from self_attention_cases import Packed

pytestmark = pytest.mark.gpu

# Heads of a multiple of 8 whose pieces behind d are zeros in LDS, those of other widths through registers, and such with rows that are not at multiples of 16 bytes.
WIDTHS = [8, 16, 24, 40, 48, 56, 72, 88, 104, 112, 120] + [4, 10, 30, 34, 42, 50, 58, 62, 66, 74, 82, 94, 106, 114, 122]
MASKS = {"causal": dict(rows=[200, 3, 66], behind=5), "window": dict(rows=[330, 40], window=150, before=1), "whole": dict(rows=[140, 1, 70], causal=False)}


def check(c):
    dev = c.inputs()
    O, lse = c.forward(dev)
    c.check_forward(O, lse)
    c.check_backward(O, lse, c.backward(O, lse, dev))


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("d", WIDTHS)
def test_every_width(d, mask):
    check(Packed(H=4, Hk=2, d=d, seed=d, **MASKS[mask]))


@pytest.mark.parametrize("d", [32, 40, 64, 96, 104, 128])
@pytest.mark.parametrize("gap", [2, 8, 14])
def test_strided_rows_of_aligned_heads(d, gap):
    check(Packed(rows=[130, 70], H=2, Hk=1, d=d, gap=gap))


@pytest.mark.parametrize("d", [34, 50, 62, 56, 126])
def test_pieces_of_odd_widths(d):
    """Few tiles of tokens with many stages, whose work is cut and joined."""
    check(Packed(rows=[300, 5, 400], H=16, Hk=1, d=d, window=90))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n", [7, 8, 9, 20, 62, 63, 64, 65])
def test_numbers_of_sequences(n, causal):
    """Up to 8 in order of length, up to 63 by one load, more by a search; empty and long ones among them."""
    rows = [(0, 1, 64, 129, 17, 0, 33, 257)[(5 * i + i // 8) % 8] for i in range(n)]
    check(Packed(rows=rows, H=2, Hk=1, d=32, causal=causal, before=2, behind=140, seed=n))


@pytest.mark.parametrize("d", [40, 50, 62, 104, 120])
def test_values_that_are_not_finite_at_other_widths(d):
    """An infinity among values that some rows do not see, a NaN in a hidden gradient's row: other rows and sequences as without them."""
    def case():
        return Packed(rows=[100, 40], H=2, Hk=1, d=d, seed=3)
    bad, clean = case(), case()
    bad.v[50, 0, 3], clean.v[50, 0, 3] = float("inf"), 0.0
    (O, lse), (Oc, lsec) = bad.forward(), clean.forward()
    assert not torch.isfinite(O[50:100, :, 3].float()).any()
    O[50:100, :, 3] = Oc[50:100, :, 3]
    clean.check_forward(O, lse)
    bad, clean = case(), case()
    bad.do[60, 1], clean.do[60, 1] = float("nan"), 0.0
    O, lse = clean.forward()
    out, want = bad.backward(O, lse), clean.backward(O, lse)
    assert out[0][60, 1].isnan().all()
    for x, y, rows in zip(out, want, ((60, 1), (slice(0, 61), 0), (slice(0, 61), 0))):
        x[rows] = y[rows]
        assert torch.isfinite(x.float()).all()
    clean.check_backward(O, lse, out)
