"""Tree rounds and forks of a context at their limits: token counts near 2^31, the last tokens of a generation."""
import numpy as np
import pytest

import synth
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


@pytest.mark.parametrize("n", [15, 63])
def test_trees_up_to_the_last_token(n):
    """With the positions that a generation of the library's own drafts needs and no more, trees that reach far past the last token are verified up to it."""
    dl, cfg, ctx, prompt = make(TINY_GQA, gen=48, max_seq=TINY_GQA.max_seq)
    want, margins = plain_stream(ctx, 0, prompt, 48)
    rng = np.random.default_rng(n)
    out = ctx.prefill(1, prompt, 48).emitted()
    while len(out) < 48:
        left = 48 - len(out)
        if left < 20:                                            # a chain, right for some steps, and then a tree that follows it
            good = want[len(out):]
            good = good[:int(rng.integers(0, 5))]
            tokens = [int(t) for t in good] + [int(t) for t in rng.integers(0, cfg.vocab, n - len(good))]
            parents = [i - 1 if i <= left else int(rng.integers(left, i)) for i in range(n)]
            got, expect = ctx.verify_tree(1, tokens, parents), min(len(good) + 1, left)
        else:
            got, expect = ctx.verify_tree(1, [], []), 1
        if not agrees(got, want, margins, len(out)):
            break
        assert expect <= len(got) <= left
        out += got
    assert len(out) > 40
    if len(out) == 48:
        with pytest.raises(dl.DelError) as e:
            ctx.verify_tree(1, [1], [-1])
        assert e.value.code == dl.ESTATE
    ctx.close()


def test_drafts_that_are_left_out_do_not_count():
    """A draft too deep to be emitted, and what follows it, may stand anywhere in the list: the others give what they give without it."""
    dl, cfg, ctx, prompt = make(TINY_GQA, gen=30)
    want, margins = plain_stream(ctx, 0, prompt, 30)
    ctx.prefill(1, prompt, 4)                                    # three tokens are left: drafts of depth 1 and 2 can be emitted
    a, b, c = (int(t) for t in want[1:4])
    wrong = (a + 1) % cfg.vocab
    tokens, parents = [wrong, 5, 6, a, 7, 8, b, 9, c, 10], [-1, 0, 1, -1, 2, 3, 3, 5, 6, 7]
    got = ctx.verify_tree(1, tokens, parents)
    if agrees(got, want, margins, 1):
        assert got == [a, b, c]
    ctx.close()


# heads whose trees of 49 nodes and more take the tcgen05 form of the tree attention in every layer, as four tiles of 16 rows for each of them
# do not fit the device at once (head dimension 128: between tcgen05 layer GEMMs; between streaming ones behind 4000 positions)
WIDE = [synth.small_variant(TINY_GQA, name="wide_hd128", n_layers=3, n_heads=40, n_kv_heads=40, head_dim=128, e_max=2, seed=91),
        synth.small_variant(TINY_GQA, name="wide_hd128_long", n_layers=3, n_heads=40, n_kv_heads=40, head_dim=128, e_max=2, prompt_len=4100, seed=93),
        synth.small_variant(TINY_GQA, name="wide_hd64", n_layers=3, n_heads=80, n_kv_heads=80, head_dim=64, e_max=2, seed=92)]


@pytest.mark.parametrize("cfg", WIDE, ids=lambda c: c.name)
@pytest.mark.parametrize("flags", ["default", "streaming head", "tcgen05 layers"])
def test_wide_trees_on_tcgen05_emit_the_plain_stream(cfg, flags):
    """Rounds whose attention runs on tcgen05 between the layer GEMMs of either form; with 16 nodes now and then, which take the other form."""
    dl, cfg, ctx, prompt = make(cfg, gen=80)
    if flags == "streaming head":
        ctx.set_flags(dl.FLAG_PDL)
    elif flags == "tcgen05 layers":
        ctx.set_flags(dl.FLAG_PDL | dl.FLAG_TC | dl.FLAG_TC_ROWS_ALL)
    want, margins = plain_stream(ctx, 0, prompt, 80)
    rng = np.random.default_rng(5)
    out, most, rounds = ctx.prefill(1, prompt, 80).emitted(), 0, 0
    while len(out) < 80:
        n = (63, 48, 16, 55)[rounds % 4]
        tokens, parents, depth = random_tree(rng, n, want[len(out):], cfg.vocab, 0.2)
        if rounds % 5 == 4:
            got, expect = ctx.round()[1].emitted(), None
        else:
            got, expect = ctx.verify_tree(1, tokens, parents), min(depth + 1, 80 - len(out))
        if not agrees(got, want, margins, len(out)):
            break
        assert expect is None or len(got) >= expect
        assert ctx.committed_len(1) == len(prompt) + len(out) + len(got) - 1
        most, rounds = max(most, len(got)), rounds + 1
        out += got
    assert rounds > 3 and most > 3, (rounds, most)
    ctx.close()
