"""Compaction in place over many rounds of pages: what is requested ahead was not yet written over, and what is written was read."""
import numpy as np
import pytest
import torch

import branch_ref as br
import paper_2504_05598_b200 as dl

pytestmark = pytest.mark.gpu


def sources(kind, start, n, rng):
    """n ascending positions, the i-th at start + i or behind it."""
    if kind == "next":                                            # one dropped in front: every source is the next slot
        step = np.ones(n, dtype=np.int64)
        step[0] = 2
    elif kind == "identity and next":                             # nothing moves for a while, then everything by one, then by two
        step = np.ones(n, dtype=np.int64)
        step[n // 3], step[2 * n // 3] = 2, 2
    elif kind == "nine of ten":
        step = 1 + (rng.random(n) < 0.1)
    elif kind == "pages":                                         # whole pages dropped: source pages are destinations of the rounds around
        step = np.where(np.arange(n) % 64 == 5, 17, 1)
    else:                                                         # dense stretches, and ones with up to 16 source pages per destination page
        step = np.where(np.arange(n) // 50 % 2 == 1, rng.integers(8, 24, n), rng.integers(1, 3, n))
    return start - 1 + np.cumsum(step)


@pytest.mark.parametrize("layers,nkv,hd", [(2, 3, 128), (3, 2, 64)])
@pytest.mark.parametrize("kind", ["next", "identity and next", "nine of ten", "pages", "dense and sparse"])
def test_many_rounds_in_place(kind, layers, nkv, hd):
    rng = np.random.default_rng(len(kind))
    starts, counts = [0, 7, 16, 31], [701, 650, 64, 333]          # up to 45 pages of destinations, 12 rounds of four
    src = torch.zeros(4, 701, dtype=torch.int32)
    for b, (s, n) in enumerate(zip(starts, counts)):
        src[b, :n] = torch.from_numpy(sources(kind, s, n, rng))
        src[b, n:] = -1
    need = [int(src[b, :n].max()) + 1 for b, n in enumerate(counts)]
    n_pages = sum(-(-x // 16) for x in need) + 2
    k, v = br.pool(n_pages, layers, nkv, hd, 3)
    table = br.tables(need, -(-max(need) // 16), n_pages, 4)
    k0, v0, args = k.cuda(), v.cuda(), (table.cuda(), src.cuda(), torch.tensor(counts, dtype=torch.int32).cuda())
    start = torch.tensor(starts, dtype=torch.int32)
    start_d = start.cuda()
    br.compact_ref(k, v, table, src, torch.tensor(counts), table, start)
    want_k, want_v, flush = k.cuda(), v.cuda(), torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    for _ in range(8):
        kd, vd = k0.clone(), v0.clone()
        flush.zero_()
        dl.kv_compact(kd, vd, args[0], args[1], args[2], args[0], start_d)
        assert torch.equal(kd, want_k) and torch.equal(vd, want_v)


def test_what_in_place_moves_leave_alone():
    """Sources outside the table or on no page, destinations on no page: nothing of theirs is written, the rest moves."""
    layers, nkv, hd, n = 1, 2, 128, 400
    k, v = br.pool(40, layers, nkv, hd, 6)
    table = br.tables([600], 38, 40, 2)
    src = torch.from_numpy(sources("nine of ten", 3, n, np.random.default_rng(0))).to(torch.int32)[None].contiguous()
    table[0, 5], table[0, 17] = -1, 40
    kd, vd, t = k.cuda(), v.cuda(), table.cuda()
    one = torch.tensor([n], dtype=torch.int32), torch.tensor([3], dtype=torch.int32)
    dl.kv_compact(kd, vd, t, src.cuda(), one[0].cuda(), t, one[1].cuda())
    br.compact_ref(k, v, table, src, one[0], table, one[1])
    assert torch.equal(kd.cpu(), k) and torch.equal(vd.cpu(), v)
