"""What a stack with an attention core refuses before it launches anything (no GPU needed)."""
import pytest
import torch

from paper_2602_22592_amd import binding as pq
from paper_2602_22592_amd.stack import AttentionCore, Stack

T, D = 128, 64


@pytest.mark.parametrize("row_start", [None, torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int64), torch.zeros(6, dtype=torch.int32)[::2]],
                         ids=["none", "short", "int64", "strided"])
def test_a_stack_with_a_core_wants_its_sequences_rows(monkeypatch, row_start):
    """Of both passes, before the first product: backward would else read buffers that a refused forward never filled."""
    def launched(*a, **k):
        raise AssertionError("launched before the refusal")
    core = AttentionCore(T, 2, 1, D // 2, 2, device="cpu")
    st = Stack(2, T, D, 96, 2, 8, 1, [1.0, 1.0], [1.0, 1.0], device="cpu", core=core)
    for name in ("linear_fwd", "linear_bwd", "ffn_fwd", "ffn_bwd", "glue_lincomb", "rope", "self_attn_fwd", "self_attn_bwd"):
        monkeypatch.setattr(pq, name, launched)
    x = torch.zeros((T, D), dtype=torch.bfloat16)
    with pytest.raises(pq.PQError, match="row_start"):
        st.forward(x, [{}, {}], row_start)
    with pytest.raises(pq.PQError, match="row_start"):
        st.backward(x, [{}, {}], [{}, {}], row_start)
