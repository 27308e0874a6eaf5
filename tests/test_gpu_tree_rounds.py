"""Rounds that verify a proposed tree of drafts, and sequences forked into further slots, on whole models.

The reference is the plain auto-regressive stream of the same weights, produced by the library itself (its parity with the oracle is tested
elsewhere): a tree round is right when it emits that stream, however the tree is shaped, and when the cache it leaves behind lets other
rounds go on with it.  Where the two best logits lie within 0.05, the order of sums may decide: a stream that parts there is compared no
further, one that parts anywhere else is wrong."""
import numpy as np
import pytest

import synth
from cases import TINY_GQA

pytestmark = pytest.mark.gpu

MARGIN = 0.05            # the bar below which this repository's parity tests do not compare an arg-max either


def make(cfg, batch=2, n_pages=None, max_seq=None, gen=None):
    import paper_2504_05598_b200 as dl
    from dataclasses import replace
    cfg = replace(cfg, batch=batch, gen_len=gen or cfg.gen_len)
    w = synth.make_weights(cfg)
    return dl, cfg, dl.DelContext(dl.make_shape(cfg, n_pages=n_pages, max_seq=max_seq or cfg.max_seq + 80), dl.upload_weights(w)), synth.make_prompt(cfg)


def plain_stream(ctx, seq, prompt, n):
    """n tokens one by one (no drafts), and by how much each was the best (the first: 0)."""
    out = ctx.prefill(seq, prompt, n).emitted()
    ctx.set_policy(seq, 1, 0)
    margins = [0.0]
    while len(out) < n:
        got = ctx.round()[seq].emitted()
        assert len(got) == 1
        z = np.sort(ctx.debug_logits(seq, ctx.shape.n_layers, 0))
        margins.append(float(z[-1] - z[-2]))
        out += got
    ctx.release(seq)
    return out, margins


def agrees(got, want, margins, at):
    """Whether got continues want from index `at` on; a difference has to lie at a near tie."""
    for i, (a, b) in enumerate(zip(got, want[at:])):
        if a != b:
            assert margins[at + i] < MARGIN, (at + i, a, b, margins[at + i])
            return False
    return True


def random_tree(rng, n, truth, vocab, share):
    """A tree of n drafts in which the true continuation goes `share` of the depth it could; its nodes lie anywhere."""
    parents, tokens, good = [], [], [-1]                         # good: the nodes of the true path, the root first
    for i in range(n):
        depth = len(good) - 1
        if depth < len(truth) and rng.random() < share:
            parents.append(good[-1])
            tokens.append(int(truth[depth]))
            good.append(i)
        else:
            parents.append(int(rng.integers(-1, i)) if i else -1)
            t = int(rng.integers(0, vocab))
            at = good.index(parents[-1]) if parents[-1] in good else None
            if at is not None and at < len(truth) and t == truth[at]:
                t = (t + 1) % vocab
            tokens.append(t)
    return tokens, parents, len(good) - 1


CONFIGS = [TINY_GQA, synth.CONFIGS["tiny"]]


@pytest.mark.parametrize("cfg", CONFIGS, ids=lambda c: c.name)
@pytest.mark.parametrize("flags", [None, "streaming head", "tcgen05 layers"])
def test_tree_rounds_emit_the_plain_stream(cfg, flags):
    dl, cfg, ctx, prompt = make(cfg, gen=90)
    if flags == "streaming head":
        ctx.set_flags(dl.FLAG_PDL)
    elif flags == "tcgen05 layers":
        ctx.set_flags(dl.FLAG_PDL | dl.FLAG_TC | dl.FLAG_TC_ROWS_ALL)
    want, margins = plain_stream(ctx, 0, prompt, 90)
    rng = np.random.default_rng(3)
    out = ctx.prefill(1, prompt, 90).emitted()
    most, rounds = 0, 0
    while len(out) < 90:
        n = int(rng.choice([0, 1, 2, 7, 16, 31, 40, 63]))
        tokens, parents, depth = random_tree(rng, n, want[len(out):], cfg.vocab, rng.choice([0.1, 0.4, 0.9]))
        if rounds % 4 == 3:                                      # a round of the library's own drafts in between
            got, expect = ctx.round()[1].emitted(), None
        else:
            got, expect = ctx.verify_tree(1, tokens, parents), min(depth + 1, 90 - len(out))
        if not agrees(got, want, margins, len(out)):
            break
        assert expect is None or len(got) >= expect              # (a wrong draft may be right by chance)
        assert ctx.committed_len(1) == len(prompt) + len(out) + len(got) - 1
        most, rounds = max(most, len(got)), rounds + 1
        out += got
    assert rounds > 4 and most > 3, (rounds, most)
    ctx.close()


def test_tree_round_keeps_the_caches_rows():
    """After a tree round the cache holds at every committed position what rounds without drafts put there.  Either may be 2e-2 of a
    row's largest value off the oracle (the bound of this repository's parity tests), so the two 4e-2 off one another."""
    dl, cfg, ctx, prompt = make(TINY_GQA, gen=40)
    want, margins = plain_stream(ctx, 0, prompt, 40)
    ctx.prefill(1, prompt, 40)
    tokens, parents, depth = random_tree(np.random.default_rng(1), 50, want[1:], cfg.vocab, 0.3)
    got = ctx.verify_tree(1, tokens, parents)
    n = len(got) if agrees(got, want, margins, 1) else 0
    assert n >= depth + 1 > 4
    keep, first = ctx.committed_len(1), len(prompt) - 2
    rows = {(layer, pos): ctx.get_kv(1, layer, pos) for layer in range(1, cfg.n_layers + 1) for pos in range(first, keep)}
    ctx.release(1)
    ctx.prefill(0, prompt, 40)
    ctx.set_policy(0, 1, 0)
    while ctx.committed_len(0) < keep:
        ctx.round()
    for (layer, pos), got in rows.items():
        for a, b in zip(got, ctx.get_kv(0, layer, pos)):
            assert np.abs(a - b).max() <= 4e-2 * np.abs(b).max() + 1e-6, (layer, pos)
    ctx.close()


def test_tree_rounds_refuse():
    dl, cfg, ctx, prompt = make(TINY_GQA, gen=20, max_seq=len(synth.make_prompt(TINY_GQA)) // 16 * 16 + 48)
    with pytest.raises(dl.DelError) as e:
        ctx.verify_tree(0, [1], [-1])
    assert e.value.code == dl.ESTATE
    ctx.prefill(0, prompt, 20)
    for tokens, parents in (([cfg.vocab], [-1]), ([-1], [-1]), ([1, 1], [-1, 1]), ([1], [-2]), ([1] * 64, [-1] * 64), ([1, 2], [-1])):
        with pytest.raises(dl.DelError) as e:
            ctx.verify_tree(0, tokens, parents)
        assert e.value.code == dl.EINVAL
    with pytest.raises(dl.DelError) as e:                        # more nodes than the sequence has positions
        ctx.verify_tree(0, [1] * 63, [-1] * 63)
    assert e.value.code == dl.ENOSPC
    ctx.draft(0, 1, 1)
    with pytest.raises(dl.DelError) as e:
        ctx.verify_tree(0, [1], [-1])
    assert e.value.code == dl.ESTATE
    ctx.verify(0)
    ctx.layer_accept(0)
    assert len(ctx.verify_tree(0, [], [])) == 1
    ctx.set_sampling(0, 0.7, 0.9, 1)
    with pytest.raises(dl.DelError) as e:
        ctx.verify_tree(0, [1], [-1])
    assert e.value.code == dl.ESTATE
    ctx.set_sampling(0, 0.0, 1.0, 0)
    left = 20 - (ctx.committed_len(0) - len(prompt) + 1)
    while left:
        left -= len(ctx.verify_tree(0, [5, 6], [-1, 0]))
    with pytest.raises(dl.DelError) as e:                        # all tokens are there
        ctx.verify_tree(0, [1], [-1])
    assert e.value.code == dl.ESTATE
    ctx.close()


def run_slots(ctx, slots, n):
    out = {s: [] for s in slots}
    while any(len(v) < n for v in out.values()):
        for s, o in enumerate(ctx.round()):
            if s in out:
                out[s] += o.emitted()
    return out


@pytest.mark.parametrize("extra", [0, 5, 16])
def test_forks_continue_the_same_stream(extra):
    """Every copy emits what the original does; the original may be released first; pages come back once nobody holds them."""
    dl, cfg, ctx, prompt = make(TINY_GQA, batch=3, gen=60)
    prompt = np.concatenate([prompt, prompt])[: len(prompt) // 16 * 16 + extra]
    want, margins = plain_stream(ctx, 0, prompt, 50)
    for turn in range(3):                                        # pages that were not given back would run out
        head = ctx.prefill(0, prompt, 50).emitted()
        for _ in range(3):
            head += ctx.round()[0].emitted()
        for s in (1, 2):
            ctx.fork(0, s, 50 - len(head))
            assert ctx.committed_len(s) == ctx.committed_len(0)
            for layer in (1, cfg.n_layers):
                for pos in range(ctx.committed_len(0)):
                    assert all(np.array_equal(a, b) for a, b in zip(ctx.get_kv(0, layer, pos), ctx.get_kv(s, layer, pos)))
            assert all(np.array_equal(a, b) for a, b in zip(ctx.get_stats(0), ctx.get_stats(s)))
            assert all(np.array_equal(a, b) for a, b in zip(ctx.get_conf_stats(0), ctx.get_conf_stats(s)))
        if turn == 1:
            ctx.release(0)
        out = run_slots(ctx, (1, 2), 50 - len(head))
        for s in (1, 2):
            agrees(head + out[s], want, margins, 0)
        for s in range(3):
            ctx.release(s)
    ctx.close()


def test_forks_with_few_pages():
    """A fork needs one page at most; without a free one it is refused and nothing changes; forked slots are full sequences."""
    prompt = np.arange(40, dtype=np.int32) % TINY_GQA.vocab
    need = 3                                                     # pages of 41 positions
    dl, cfg, ctx, _ = make(TINY_GQA, batch=3, gen=30, n_pages=16, max_seq=320)
    ctx.prefill(0, prompt, 20)
    ctx.prefill(1, np.arange(16 * (16 - need) - 1, dtype=np.int32) % cfg.vocab, 2)
    with pytest.raises(dl.DelError) as e:
        ctx.fork(0, 2, 5)
    assert e.value.code == dl.ENOSPC
    ctx.fork(0, 1, 19)                                           # the pages of slot 1 itself are given up for it
    assert ctx.committed_len(1) == 40
    out = run_slots(ctx, (0, 1), 19)
    first, margins = plain_stream(ctx, 2, prompt, 20)
    agrees(out[0], first, margins, 1)
    agrees(out[1], first, margins, 1)
    for args in ((0, 0, 5), (0, 3, 5), (-1, 1, 5), (0, 1, 0)):
        with pytest.raises(dl.DelError) as e:
            ctx.fork(*args)
        assert e.value.code == dl.EINVAL
    ctx.release(0)
    with pytest.raises(dl.DelError) as e:
        ctx.fork(0, 1, 5)
    assert e.value.code == dl.ESTATE
    ctx.close()


def test_sampled_forks_go_their_own_ways():
    """Slots with seeds of their own draw different answers from one prompt; with the same seed, the same one."""
    dl, cfg, ctx, prompt = make(TINY_GQA, batch=3, gen=30)
    ctx.prefill(0, prompt, 30)
    for s, seed in ((0, 1), (1, 1), (2, 2)):
        ctx.set_sampling(s, 1.0, 1.0, seed)
    ctx.fork(0, 1, 29)
    ctx.fork(0, 2, 29)
    out = run_slots(ctx, (0, 1, 2), 29)
    assert out[0] != out[2]
    # the uniform numbers are the same; a near tie of a cumulative sum is the only way for 0 and 1 to part
    same = next((i for i, (a, b) in enumerate(zip(out[0], out[1])) if a != b), 29)
    assert same >= 5
    ctx.close()
