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


FAR = dict(table=1 << 32, lens=2 << 32, parents=3 << 32, spare=4 << 32, n_spare=5 << 32, new_table=6 << 32, new_lens=7 << 32, free_pages=8 << 32, counts=9 << 32)
BYTES = dict(table=32, lens=8, parents=8, spare=16, n_spare=4, new_table=32, new_lens=8, free_pages=32, counts=8)       # of refusals.FORK


@pytest.mark.parametrize("out", ["new_table", "new_lens", "free_pages", "counts"])
@pytest.mark.parametrize("other", list(FAR))
def test_fork_refuses_to_write_what_it_reads_or_writes(out, other):
    """The last word of the one on the first of the other, the first on the last."""
    if out == other:
        return
    for at in (FAR[other] - BYTES[out] + 4, FAR[other] + BYTES[other] - 4):
        assert refusals.call("del_kv_fork", dl.ForkC, refusals.FORK, dict(FAR, **{out: at})) == dl.EINVAL
