"""Operators of branching decoding, on the host: further calls that are refused (no kernel is launched here)."""
import pytest
import torch

import paper_2504_05598_b200 as dl
import test_branching_refusals as refusals


@pytest.mark.parametrize("scale", [0.0, 0, -0.0, 1e-50, -0.5, 1e39, float("inf"), float("nan")])
def test_binding_refuses_a_scale_that_is_no_positive_fp32_number(scale):
    """Zero is the C call's word for the default: handed on, it would give other scores than the ones asked for."""
    k, v = torch.zeros(4, 1, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(4, 1, 2, 64, 16, dtype=torch.bfloat16)
    table = torch.zeros(1, 4, dtype=torch.int32)
    with pytest.raises(dl.DelError, match="scale") as e:
        dl.tree_attention(torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16), k, v, 1, table, table[0, :1], scale=scale)
    assert e.value.code == dl.EINVAL


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38])
def test_tree_attention_refuses_a_scale_whose_product_with_log2_e_is_infinite(scale):
    """Scores of zero would be no numbers."""
    assert refusals.call("del_tree_attention", dl.TreeAttnC, refusals.TREE, dict(scale=scale)) == dl.EINVAL
