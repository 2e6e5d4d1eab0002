"""CPU tests of the attention module's construction."""
import pytest
import torch

from paper_2607_20652_gb300.attention import Attention


@pytest.mark.parametrize("context", [0, None])
def test_without_a_context_there_are_no_positions(context):
    m = Attention(64, 4, context=context)
    assert m.cos is None and m.sin is None
    assert [n for n, _ in m.named_parameters()] == ["q_norm", "k_norm", "qkv.weight", "out.weight"]


def test_tables_reach_the_context_and_stay_in_fp32():
    m = Attention(64, 4, context=10).to(torch.bfloat16)
    assert m.cos.shape == (10, 8) and m.cos.dtype == m.sin.dtype == torch.float32 and m.q_norm.dtype == torch.bfloat16
    assert "cos" not in m.state_dict()
    with pytest.raises(ValueError):
        Attention(64, 4, 3)
    with pytest.raises(ValueError):
        Attention(60, 4)
