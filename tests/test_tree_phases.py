"""The barriers of the tcgen05 tree attention in a model on the host: no order of events lets the softmax warps read or rescale an output
that MMAs still write, and none leaves a role waiting for good.

The model has the roles of csrc/tree_attn_tc.cu: keys and values of a block arrive at any time; the MMA warp waits and issues in its
program order; MMAs run in that order; a tile's softmax warps (which move together here) wait for their scores, perhaps rescale the
output, hand over their probabilities, and behind the last block wait until the output is complete.  A barrier is the number of its completed phases; a wait
by parity p passes where the parity of the phase in progress is not p.  All reachable states are visited."""
import os
import re

import pytest

from paper_2504_05598_b200 import build


def passes(completed, parity):
    return completed & 1 != parity


def explore(n, tiles, end):
    """(an output was touched too early, some state has no way on) over all orders of events for n blocks; `end`: how the softmax warps
    wait behind the last block ("own barrier": one that the MMA warp commits to once; else the product barrier's phases, in turn)."""
    program = [("s", 0, t) for t in range(tiles)]               # ("s" or "p", block, tile): scores, products
    for j in range(n):
        if tiles == 1:
            program += ([("s", j + 1, 0)] if j + 1 < n else []) + [("p", j, 0)]
        else:
            for t in range(tiles):
                program += [("p", j, t)] + ([("s", j + 1, t)] if j + 1 < n else [])

    def buf(j, t):
        return t if tiles == 2 else j & 1

    def phase(j):                                                # of a score buffer's barriers in block j
        return j if tiles == 2 else j >> 1

    own = end == "own barrier"
    softmax = [s for j in range(n) for s in (("scores", j), ("hand over", j))] + ([("all", 0)] if own else [("phase", j) for j in end])
    # blocks whose keys, whose values have arrived; MMAs issued, done; each tile's softmax warps: steps taken
    start = (0, 0, 0, 0, (0,) * tiles)
    seen, todo, early, stuck = {start}, [start], False, False
    while todo:
        state = todo.pop()
        keys, values, issued, done, at = state
        s_full = [sum(1 for k, j, t in program[:done] if k == "s" and buf(j, t) == b) for b in range(2)]
        o_done = [sum(1 for k, j, t in program[:done] if k == "p" and t == tile) for tile in range(tiles)]
        p_full = [0, 0]
        for tile in range(tiles):
            for j in range(n):
                p_full[buf(j, tile)] += at[tile] > 2 * j + 1
        nexts = []
        if keys < n:
            nexts.append((keys + 1, values, issued, done, at))
        if values < n:
            nexts.append((keys, values + 1, issued, done, at))
        if issued < len(program):
            kind, j, t = program[issued]
            if (kind == "s" and keys > j) or (kind == "p" and values > j and passes(p_full[buf(j, t)], phase(j) & 1)):
                nexts.append((keys, values, issued + 1, done, at))
        if done < issued:
            nexts.append((keys, values, issued, done + 1, at))
        for t in range(tiles):
            if at[t] == len(softmax):
                early |= o_done[t] < n                           # the output is read
                continue
            kind, j = softmax[at[t]]
            on = keys, values, issued, done, at[:t] + (at[t] + 1,) + at[t + 1:]
            if kind == "scores":
                if passes(s_full[buf(j, t)], phase(j) & 1):
                    nexts.append(on)
            elif kind == "hand over":
                nexts.append(on)                                 # without rescaling; with it, once the block before is part of the output:
                if j and (tiles == 2 or passes(o_done[t], (j - 1) & 1)):
                    early |= o_done[t] < j
            elif kind == "all":
                if o_done[t] == n:
                    nexts.append(on)
            elif passes(o_done[t], j & 1):
                nexts.append(on)
        if not nexts and not all(a == len(softmax) for a in at):
            stuck = True
        for s in nexts:
            if s not in seen:
                seen.add(s)
                todo.append(s)
    return early, stuck


@pytest.mark.parametrize("n,tiles", [(n, 1) for n in range(1, 8)] + [(n, 2) for n in range(1, 5)])
def test_no_output_is_touched_early(n, tiles):
    assert explore(n, tiles, "own barrier") == (False, False)


@pytest.mark.parametrize("n", range(2, 8))
def test_phases_of_the_product_barrier_do_not_tell(n):
    """With one tile the last phase alone passes while the one before it is open, and a wait for that one first blocks where both are over."""
    assert explore(n, 1, [n - 1]) == (True, False)
    assert explore(n, 1, [n - 2, n - 1])[1]


def test_the_kernel_ends_on_the_barrier_of_the_model():
    with open(os.path.join(build.CSRC, "tree_attn_tc.cu")) as f:
        source = f.read()
    end = source[source.index("mbar_arrive(&p_full[buf])"):]
    assert re.findall(r"wait_or_err\(&(\w+)\[", end) == ["o_all"]
    assert len(re.findall(r"umma_commit\(&o_all\[t\]\)", source)) == 1 and "if (j == n_kb - 1) umma_commit(&o_all[t]);" in source
