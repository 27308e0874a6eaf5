"""Forks without spare pages to hand out: an empty list is no error where no page is wanted, and none is missing."""
import pytest
import torch

import branch_ref as br
import paper_2504_05598_b200 as dl
from test_gpu_branching import run_fork

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("count", [0, 3])
def test_fork_with_an_empty_list_of_spare_pages(count):
    k, v = br.pool(8, 1, 2, 64, 2)
    table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32)
    lens = torch.tensor([32, 20], dtype=torch.int32)
    mine = run_fork(k, v, table, lens, [1, 0, 0], [], count, 2, 0)              # reordered, full pages shared: no page is wanted
    assert mine[0].tolist() == [[2, 3], [0, 1], [0, 1]] and mine[2].tolist() == [4, 0]
    mine = run_fork(k, v, table, lens, [1, 1], [], count, 3, 1)                  # one copy is wanted
    assert mine[2].tolist()[1] == 1
