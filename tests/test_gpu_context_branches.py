"""Tree rounds and forks of a context at their limits: token counts near 2^31, the last tokens of a generation."""
import numpy as np
import pytest

from cases import TINY_GQA
from test_gpu_tree_rounds import agrees, make, plain_stream, random_tree

pytestmark = pytest.mark.gpu


def test_token_counts_are_added_in_64_bits():
    """A count of tokens that reaches past 32 bits with the positions before it is too many, not few."""
    dl, cfg, ctx, prompt = make(TINY_GQA, gen=20)
    ctx.prefill(0, prompt, 20)
    for n in (2 ** 31 - 1, 2 ** 31 - 20, 10 ** 6):
        for call in (lambda: ctx.fork(0, 1, n), lambda: ctx.prefill(1, prompt, n)):
            with pytest.raises(dl.DelError) as e:
                call()
            assert e.value.code == dl.ENOSPC
    ctx.fork(0, 1, 19)
    assert ctx.committed_len(1) == len(prompt)
    ctx.close()
