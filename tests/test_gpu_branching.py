"""Operators of branching decoding on the GPU against their plain 64-bit forms."""
import numpy as np
import pytest
import torch

import branch_ref as br
import paper_2504_05598_b200 as dl

pytestmark = pytest.mark.gpu
CANARY = 7.0


def dev(t):
    return None if t is None else t.cuda()


# ---------------------------------------------------------------- tree attention
def check_tree(q, k, v, layer, table, lens, nodes, mask, scale=None, low=False, max_len=0):
    """Both forms of the kernel: calls of this size take the mma.sync one, and with a table of 4096 columns (whose further entries name no
    page) and no word about the lengths, the tcgen05 one, with parts of the keys that have nothing to do."""
    wide = torch.full((table.shape[0], 4096), 0x7ffffff0, dtype=torch.int32)
    wide[:, : table.shape[1]] = table
    check_tree_once(q, k, v, layer, wide, lens, nodes, mask, scale, low)
    return check_tree_once(q, k, v, layer, table, lens, nodes, mask, scale, low, max_len)


def check_tree_once(q, k, v, layer, table, lens, nodes, mask, scale=None, low=False, max_len=0):
    """Runs the operator on canary-filled outputs and holds every element to its bound."""
    ref, mass, dots = br.tree_attention_ref(q, k, v, layer, table, lens, nodes, mask, scale)
    out = torch.full(q.shape, CANARY, dtype=torch.bfloat16, device="cuda")
    out_lo = torch.full(q.shape, CANARY, dtype=torch.bfloat16, device="cuda") if low else None
    dl.tree_attention(q.cuda(), k.cuda(), v.cuda(), layer, table.cuda(), lens.cuda(), dev(nodes), dev(mask), out=out, out_lo=out_lo, scale=scale, max_len=max_len)
    got = out.cpu().double()
    idle = ref.isnan().all(-1)
    for b in range(q.shape[0]):                                   # rows behind the last node: untouched
        live = q.shape[1] if nodes is None else min(max(int(nodes[b]), 0), q.shape[1])
        assert (got[b, live:] == CANARY).all()
        idle[b, :live] = False
    if low:
        assert (out_lo.cpu()[idle] == CANARY).all()
        got = torch.where(idle[..., None], got, got + out_lo.cpu().double())
    bad = ref.isnan() & ~idle[..., None]
    assert (got.isnan() == bad)[~idle].all()
    fine = ~ref.isnan()
    bound = br.tree_attention_bound(ref, mass, dots, q.shape[3], k.shape[0] * 16, low)
    inf = fine & ref.isinf()
    assert (got[inf] == ref[inf]).all()
    fine &= ~ref.isinf()
    worst = ((got - ref).abs() / bound)[fine].max() if fine.any() else 0
    assert worst <= 1, float(worst)
    return out


def make_tree(nh, nkv, hd, lens, nodes, n, seed=0, layers=2, extra=3, mask=True, cols=None):
    batch = len(lens)
    need = [a + b for a, b in zip(lens, nodes)]
    n_pages = sum(-(-x // 16) for x in need) + extra
    k, v = br.pool(n_pages, layers, nkv, hd, seed)
    table = br.tables(need, cols or max(1, -(-max(need) // 16)), n_pages, seed + 1)
    g = torch.Generator().manual_seed(seed + 2)
    q = (1.5 * torch.randn(batch, n, nh, hd, generator=g)).to(torch.bfloat16)
    m = br.random_masks(batch, n, seed + 3) if mask else None
    return q, k, v, table, torch.tensor(lens, dtype=torch.int32), torch.tensor(nodes, dtype=torch.int32), m


HEADS = [(4, 4, 64), (32, 8, 64), (8, 2, 128), (5, 5, 128), (6, 1, 128), (12, 1, 64)]


@pytest.mark.parametrize("nh,nkv,hd", HEADS)
@pytest.mark.parametrize("n", [1, 5, 16, 33, 64])
def test_tree_attention(nh, nkv, hd, n):
    lens = [0, 1, 15, 16, 129, 200]
    nodes = [n, max(1, n // 2), n, 0, n, 1]
    q, k, v, table, lens, nodes, m = make_tree(nh, nkv, hd, lens, nodes, n, seed=n)
    for layer in (1, 2):
        check_tree(q, k, v, layer, table, lens, nodes, m, low=layer == 2)


@pytest.mark.parametrize("nh,nkv,hd,n", [(8, 2, 128, 3), (4, 4, 64, 17), (8, 2, 128, 40), (32, 8, 64, 26)])
def test_tree_attention_long(nh, nkv, hd, n):
    q, k, v, table, lens, nodes, m = make_tree(nh, nkv, hd, [2500, 1203], [n, n - 1], n, seed=5, layers=1)
    check_tree(q, k, v, 1, table, lens, nodes, m, max_len=2500)
    check_tree(q, k, v, 1, table, lens, nodes, m, max_len=100)           # a bound that does not hold only splits badly
    check_tree(q, k, v, 1, table, lens, None, None, scale=0.31)          # a chain in every sequence (its last nodes lie behind the table)


@pytest.mark.parametrize("hd,n", [(64, 1), (128, 1), (64, 40), (128, 40)])
def test_tree_attention_strides(hd, n):
    """Queries and outputs as slices of wider rows, a table and pages in use by others."""
    nh, nkv = 8, 2
    q, k, v, table, lens, nodes, m = make_tree(nh, nkv, hd, [37, 64, 5], [n, n, n], n, seed=9)
    width = (nh + 2 * nkv) * hd
    fused = torch.zeros(3, n + 2, width, dtype=torch.bfloat16, device="cuda")
    qs = fused[:, 1:n + 1, : nh * hd].unflatten(2, (nh, hd))
    qs.copy_(q)
    wide = torch.full((3, n, 2, nh, hd), CANARY, dtype=torch.bfloat16, device="cuda")
    tab = torch.full((3, table.shape[1] + 5), -7, dtype=torch.int32)
    tab[:, : table.shape[1]] = table
    want = check_tree(q, k, v, 1, table, lens, nodes, m)
    dl.tree_attention(qs, k.cuda(), v.cuda(), 1, tab.cuda()[:, : table.shape[1]], lens.cuda(), nodes.cuda(), m.cuda(), out=wide[:, :, 1])
    assert torch.equal(wide[:, :, 1], want)
    assert (wide[:, :, 0] == CANARY).all()


@pytest.mark.parametrize("nh,nkv,hd", [(8, 2, 64), (8, 2, 128), (32, 4, 128)])
@pytest.mark.parametrize("n", [2, 9, 40])
def test_what_is_masked_never_counts(nh, nkv, hd, n):
    """NaN and infinities in slots that nobody may see, and in drafted tokens that some rows see."""
    q, k, v, table, lens, nodes, m = make_tree(nh, nkv, hd, [0, 21, 35], [n, n, n - 1], n, seed=11)
    m &= ~(1 << (n - 1))                                         # nobody sees the last node, not even itself
    m[:, 0] = 0                                                  # the first row sees committed positions alone
    for b in range(3):
        for p in range(int(lens[b]) + int(nodes[b]), table.shape[1] * 16):      # never written
            if 0 <= int(table[b, p // 16]) < k.shape[0]:
                k[int(table[b, p // 16]), :, :, p % 16] = float("nan")
                v[int(table[b, p // 16]), :, :, :, p % 16] = float("inf")
        p = int(lens[b]) + n - 1
        if n <= int(nodes[b]):
            k[int(table[b, p // 16]), :, :, p % 16] = float("inf")
            v[int(table[b, p // 16]), :, :, :, p % 16] = float("nan")
        p = int(lens[b])                                          # the root's values: infinite in one dimension, for those that see it
        v[int(table[b, p // 16]), :, :, 3, p % 16] = float("inf")
    check_tree(q, k, v, 2, table, lens, nodes, m)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("batch", [12, 40])
def test_many_sequences_of_many_rows(hd, batch):
    """160 rows per kv head in so many sequences (most of them without nodes) that a CTA of the tcgen05 form takes two tiles: with the
    keys in parts (12), and as a whole (40).  Slots that nobody sees and some drafted tokens hold no numbers, a page is named wrongly."""
    n = 40
    q, k, v, table, lens, nodes, m = make_tree(8, 2, hd, [0, 700, 35, 301] + [0] * (batch - 4), [n, n, n - 1, 17] + [0] * (batch - 4), n, seed=41)
    m &= ~(1 << (n - 1))
    m[:, 0] = 0
    for b in range(4):
        end = int(lens[b]) + int(nodes[b])
        for p in range(end, -(-end // 16) * 16):
            k[int(table[b, p // 16]), :, :, p % 16] = float("nan")
            v[int(table[b, p // 16]), :, :, :, p % 16] = float("inf")
        p = int(lens[b])
        v[int(table[b, p // 16]), :, :, 5, p % 16] = float("-inf")
        if n <= int(nodes[b]):
            p = int(lens[b]) + n - 1
            k[int(table[b, p // 16]), :, :, p % 16] = float("inf")
            v[int(table[b, p // 16]), :, :, :, p % 16] = float("nan")
    table[1, 20] = -1
    q[3, 7, 6, 9] = float("nan")
    check_tree(q, k, v, 2, table, lens, nodes, m)
    check_tree(q, k, v, 1, table, lens, nodes, m, scale=0.4, low=True)


@pytest.mark.parametrize("n", [1, 20])
@pytest.mark.parametrize("hd", [64, 128])
def test_no_number_stays_in_its_row(hd, n):
    """A NaN query, key or value gives NaN where the formula has it and nowhere else."""
    q, k, v, table, lens, nodes, m = make_tree(4, 2, hd, [40, 40], [n, n], n, seed=3)
    q[0, n - 1, 1, 5] = float("nan")
    k[int(table[1, 1]), :, 1, 7] = float("nan")
    check_tree(q, k, v, 1, table, lens, nodes, m)


@pytest.mark.parametrize("hd,n", [(64, 3), (128, 3), (64, 30), (128, 30)])
def test_tables_that_name_no_page(hd, n):
    """Page ids outside the pool and positions behind the table are masked; lens and nodes outside their ranges are cut."""
    q, k, v, table, lens, nodes, m = make_tree(4, 2, hd, [100, 50, 64], [n, n, n], n, seed=21)
    table[0, 2], table[1, 0], table[1, 3] = -1, k.shape[0], 1 << 30
    check_tree(q, k, v, 1, table, lens, nodes, m)
    check_tree(q, k, v, 1, table[:, :4], torch.tensor([64, 1 << 30, -5], dtype=torch.int32), torch.tensor([n + 9, n, -1], dtype=torch.int32), m)
    table[:] = -1
    check_tree(q, k, v, 1, table, lens, nodes, m)                # nothing to see: zeros


def test_tree_attention_of_identical_pages_is_the_mean_of_their_values():
    """Equal keys: the output is the plain mean, whatever the split."""
    for nh, n in ((2, 1), (8, 40)):
        k, v = br.pool(200, 1, 2, 128, 1)
        k[:] = 0.5
        q = torch.ones(1, n, nh, 128, dtype=torch.bfloat16)
        table = torch.arange(200, dtype=torch.int32)[None]
        check_tree(q, k, v, 1, table, torch.tensor([3199 - n], dtype=torch.int32), None, None)


# ---------------------------------------------------------------- compaction
@pytest.mark.parametrize("layers,nkv,hd", [(1, 1, 64), (3, 2, 128), (2, 5, 64)])
@pytest.mark.parametrize("shift", [0, 3, 40])
def test_compact_in_place(layers, nkv, hd, shift):
    """The accepted path of a tree moved together: sources ascend and lie behind their destinations."""
    rng = np.random.default_rng(shift)
    lens, n = [0, 5, 16, 100, 31], 90
    need = [x + n + 1 + shift for x in lens]
    n_pages = sum(-(-x // 16) for x in need) + 2
    k, v = br.pool(n_pages, layers, nkv, hd, 3)
    table = br.tables(need, -(-max(need) // 16), n_pages, 4)
    src = torch.zeros(5, 64, dtype=torch.int32)
    counts = torch.tensor([64, 1, 33, 17, 0], dtype=torch.int32)
    for b in range(5):
        path = np.sort(rng.choice(n, 64, replace=False)) if b else np.arange(64)
        src[b] = torch.from_numpy(lens[b] + shift + path)
    start = torch.tensor(lens, dtype=torch.int32)
    kd, vd = k.cuda(), v.cuda()
    dl.kv_compact(kd, vd, table.cuda(), src.cuda(), counts.cuda(), table.cuda(), start.cuda())
    br.compact_ref(k, v, table, src, counts, table, start)
    assert torch.equal(kd.cpu(), k) and torch.equal(vd.cpu(), v)


@pytest.mark.parametrize("layers,nkv,hd,n", [(2, 2, 64, 1), (1, 3, 128, 15), (2, 1, 128, 700), (1, 2, 64, 333)])
def test_compact_into_other_pages(layers, nkv, hd, n):
    """Any order, the same source twice, part-filled first pages whose other slots stay, tables and positions out of range."""
    rng = np.random.default_rng(n)
    batch, length = 3, 2 * n + 5
    old, new = -(-length // 16), -(-(n + 20) // 16)
    n_pages = batch * (old + new)
    k, v = br.pool(n_pages, layers, nkv, hd, 8)
    table = br.tables([16 * (old + new)] * batch, old + new, n_pages, 6)
    src_table, dst_table = table[:, :old].clone(), table[:, old:].clone()
    src = torch.from_numpy(rng.integers(0, length, (batch, n + 3))).to(torch.int32)
    src[0, 0], src[1, n // 2], src[2, n - 1] = -1, old * 16, 1 << 30
    src_table[1, old // 2] = n_pages
    dst_table[2, 0] = -3
    counts = torch.tensor([n, n + 3, n + 100], dtype=torch.int32)
    start = torch.tensor([0, 7, 19], dtype=torch.int32)
    kd, vd = k.cuda(), v.cuda()
    wide = torch.zeros(batch, n + 9, dtype=torch.int32, device="cuda")
    wide[:, : n + 3] = src.cuda()
    dl.kv_compact(kd, vd, table.cuda()[:, :old].copy_(src_table), wide[:, : n + 3], counts.cuda(), dst_table.cuda(), start.cuda())
    br.compact_ref(k, v, src_table, src, counts, dst_table, start)
    assert torch.equal(kd.cpu(), k) and torch.equal(vd.cpu(), v)


def test_compact_moves_bits():
    k, v = br.pool(2, 1, 1, 64, 0)
    kb, vb = k.view(torch.int16), v.view(torch.int16)
    kb[0] = torch.arange(-512, 512).view(kb[0].shape).to(torch.int16) * 64        # NaN patterns, infinities, -0 among them
    vb[0] = torch.arange(512, -512, -1).view(vb[0].shape).to(torch.int16) * 64
    kd, vd = k.cuda(), v.cuda()
    one = torch.tensor([[0]], dtype=torch.int32, device="cuda")
    src = torch.arange(16, dtype=torch.int32, device="cuda").flip(0)[None].contiguous()
    dl.kv_compact(kd, vd, one, src, torch.tensor([16], dtype=torch.int32, device="cuda"), one + 1, torch.tensor([0], dtype=torch.int32, device="cuda"))
    assert torch.equal(kd.cpu().view(torch.int16)[1], kb[0].flip(2)) and torch.equal(vd.cpu().view(torch.int16)[1], vb[0].flip(3))


# ---------------------------------------------------------------- forks
def run_fork(k, v, table, lens, parents, spare, n_spare, cols, room, free=True):
    n_new, n_pages = len(parents), k.shape[0]
    i32 = dict(dtype=torch.int32)
    parents, spare = torch.tensor(parents, **i32), torch.tensor(spare, **i32)
    mine = [torch.full((n_new, cols), -9, **i32), torch.full((n_new,), -9, **i32), torch.full((2,), -9, **i32), torch.full((n_pages,), -9, **i32) if free else None]
    theirs = [dev(t) for t in mine]
    kd, vd, count = k.cuda(), v.cuda(), torch.tensor([n_spare, 5], **i32)
    dl.kv_fork(kd, vd, table.cuda(), lens.cuda(), parents.cuda(), spare.cuda(), count.cuda(), theirs[0], theirs[1], theirs[2], room=room, free_pages=theirs[3])
    br.fork_ref(k, v, table, lens, parents, spare, count, mine[0], mine[1], mine[2], room, mine[3])
    for a, b in zip(mine, theirs):
        assert a is None or torch.equal(a, b.cpu()), (a, b)
    assert torch.equal(kd.cpu(), k) and torch.equal(vd.cpu(), v)
    return mine


@pytest.mark.parametrize("layers,nkv,hd", [(1, 1, 64), (2, 3, 128), (5, 4, 64)])
@pytest.mark.parametrize("rows,room", [(1, 0), (4, 1), (37, 17), (300, 1)])
def test_fork(layers, nkv, hd, rows, room):
    rng = np.random.default_rng(rows)
    lens = [int(x) for x in rng.integers(0, 70, rows)]
    lens[0] = 16 * (rows % 3)
    held = sum(-(-x // 16) for x in lens)
    new = rows + rows // 2
    n_pages = held + 4 * new + 3
    k, v = br.pool(n_pages, layers, nkv, hd, 1)
    perm = rng.permutation(n_pages).tolist()
    table = torch.full((rows, 6), -5, dtype=torch.int32)
    for b, x in enumerate(lens):
        for p in range(-(-x // 16)):
            table[b, p] = perm.pop()
    parents = [int(x) for x in rng.integers(-1, rows + 1, new)]
    mine = run_fork(k, v, table, torch.tensor(lens, dtype=torch.int32), parents, perm, len(perm), 7, room)
    assert mine[2][1] == 0
    run_fork(k, v, table, torch.tensor(lens, dtype=torch.int32), parents, perm, len(perm), 7, room, free=False)


def test_fork_without_enough_pages():
    """Spare pages run out, or are none: entries of -1, counted; a part-filled page that is named wrongly is not copied."""
    k, v = br.pool(20, 1, 2, 64, 2)
    table = torch.tensor([[0, 1], [2, 99], [3, 4]], dtype=torch.int32)
    lens = torch.tensor([20, 30, -4], dtype=torch.int32)
    mine = run_fork(k, v, table, lens, [0, 0, 1, 1, 0, 2, 7], [10, 500, 11, 12], 4, 4, 40)
    assert mine[2][1] > 5
    run_fork(k, v, table, lens, [0, 0, 0], [10, 11, 12], 1, 2, 0)
    run_fork(k, v, table, lens, [0, 0, 0], [10, 11, 12], -1, 2, 0)
    run_fork(k, v, table, lens, [0, 0, 0], [10, 11, 12], 99, 1, 0)       # tables of one column: rows are cut to it


def test_fork_of_1024_rows():
    k, v = br.pool(3000, 1, 1, 64, 2)
    rng = np.random.default_rng(0)
    lens = torch.from_numpy(rng.integers(0, 33, 1024)).to(torch.int32)
    table = torch.from_numpy(rng.permutation(1024 * 2).reshape(1024, 2)).to(torch.int32)
    run_fork(k, v, table, lens, [int(x) for x in rng.integers(0, 1024, 1024)], list(range(2048, 3000)), 952, 3, 1)


# ---------------------------------------------------------------- beam selection
def check_beam(logits, scores, k, finished=None, eos=0):
    batch = logits.shape[0]
    outs = [torch.full((batch, k), -77, dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32)]
    dl.beam_select(logits if logits.is_cuda else logits.cuda(), scores.cuda(), *outs, finished=dev(finished), eos=eos)
    want = br.beam_ref(logits, scores, k, finished, eos)
    assert np.array_equal(outs[1].cpu().numpy(), want[1]), (outs[1], want[1])
    assert np.array_equal(outs[2].cpu().numpy(), want[2])
    got = outs[0].cpu().double().numpy()
    inf = np.isinf(want[0])
    assert np.array_equal(np.isinf(got), inf)
    # the log-sum-exp: sums of positive fp32 numbers, each exponential within a few units of its last place and its argument
    # (x - m) log2 e within 2^-23 of its size (at most 150, behind which nothing counts); then one rounding of the score
    err = np.abs(got[~inf] - want[0][~inf])
    assert (err <= 2.0 ** -24 * np.abs(want[0][~inf]) + 150 * 2.0 ** -23).all(), err.max()
    return outs


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("batch,beams,vocab,k", [(1, 1, 1, 1), (2, 3, 7, 5), (1, 4, 100, 64), (3, 2, 1000, 4), (1, 8, 32000, 16), (2, 5, 32003, 10),
                                                 (5, 4, 8192, 8), (40, 2, 9000, 3), (1, 2, 300001, 7), (200, 1, 20000, 2), (1, 64, 257, 64)])
def test_beam_select(batch, beams, vocab, k, dtype):
    g = torch.Generator().manual_seed(vocab)
    logits = (3 * torch.randn(batch, beams, vocab, generator=g)).to(dtype)
    scores = -5 * torch.rand(batch, beams, generator=g)
    check_beam(logits, scores, k)
    finished = torch.rand(batch, beams, generator=g) < 0.4
    check_beam(logits, scores, k, finished, vocab // 2)


@pytest.mark.parametrize("vocab", [50, 5000, 70000])
def test_beam_select_orders_ties_by_index(vocab):
    """Few different values: within a row the lower token, over equal rows the lower row."""
    g = torch.Generator().manual_seed(1)
    row = torch.randint(0, 3, (vocab,), generator=g).float()
    logits = row.expand(2, 4, vocab).contiguous()
    check_beam(logits, torch.zeros(2, 4), 33)
    check_beam(torch.zeros(1, 3, vocab), torch.tensor([[-1.0, -1.0, -2.0]]), 20)
    check_beam((logits * 0 - 0.0), torch.zeros(2, 4), 5)


@pytest.mark.parametrize("vocab", [3000, 140000])
def test_beam_select_of_sorted_logits(vocab):
    """The order in which a threshold from part of the logits helps least."""
    up = torch.linspace(-9, 9, vocab)
    for row in (up, up.flip(0), torch.cat([up[::2], up[1::2]])):
        check_beam(torch.stack([row, row * 0.9]).unsqueeze(0).contiguous(), torch.tensor([[-1.0, -1.5]]), 48)


@pytest.mark.parametrize("vocab", [40, 20000])
def test_beam_select_without_numbers(vocab):
    """Masked tokens, dead beams, NaN and infinities; fewer continuations above -inf than are asked for."""
    inf, g = float("inf"), torch.Generator().manual_seed(2)
    logits = torch.randn(6, 3, vocab, generator=g)
    scores = -torch.rand(6, 3, generator=g)
    logits[0, :, 3:] = -inf                                     # three tokens allowed
    logits[1, 0, 5], logits[1, 1, 6], logits[1, 2, 7] = float("nan"), inf, -inf
    logits[2, 1] = -inf
    scores[3, 0], scores[3, 1] = -inf, float("nan")
    scores[4, 0] = inf
    logits[5] = logits[5] * 1e-3 - 1e4                          # far from zero, and one thread's share all masked
    logits[5, :, ::4] = -inf
    check_beam(logits, scores, 12)
    scores[:] = -inf
    check_beam(logits, scores, 12)
    finished = torch.ones(6, 3, dtype=torch.bool)
    scores = -torch.rand(6, 3, generator=g)
    scores[2, 1] = float("nan")
    check_beam(logits, scores, 12, finished, 2)


def test_beam_select_strides():
    """Rows that start on odd addresses, and rows further apart than they are long."""
    g = torch.Generator().manual_seed(3)
    for dtype in (torch.float32, torch.bfloat16):
        base = torch.randn(2 * 3 * 5013 + 1, generator=g).to(dtype).cuda()
        view = base[1:].view(2, 3, 5013)[:, :, :4999]
        check_beam(view, torch.zeros(2, 3), 9)


def test_beam_select_with_a_workspace():
    """A workspace that is handed in: whatever it holds, the same results; one byte too few is refused."""
    g = torch.Generator().manual_seed(9)
    for batch, beams, vocab, k in [(1, 4, 3001, 4), (30, 5, 20011, 9)]:
        logits, scores = torch.randn(batch, beams, vocab, generator=g), torch.zeros(batch, beams)
        want = check_beam(logits, scores, k)
        shape = dl.BeamC(*(dict(batch=batch, beams=beams, vocab=vocab, k=k, dtype=0, row_stride=vocab).get(n, 0) for n, _ in dl.BeamC._fields_))
        size = dl.load_library().del_beam_workspace_bytes(dl.C.byref(shape))
        outs = [torch.zeros_like(t) for t in want]
        for fill in (0, 255, 127):
            work = torch.full((size,), fill, dtype=torch.uint8, device="cuda")
            dl.beam_select(logits.cuda(), scores.cuda(), *outs, workspace=work)
            assert all(torch.equal(a, b) for a, b in zip(outs, want))
        with pytest.raises(dl.DelError) as e:
            dl.beam_select(logits.cuda(), scores.cuda(), *outs, workspace=work[:-1])
        assert e.value.code == dl.ENOSPC


# ---------------------------------------------------------------- offsets that 32 bits do not hold
def test_caches_of_more_than_2_32_elements():
    """Pages at the far end of a large cache attended (both forms), compacted and forked; the few pages in use are checked against the
    same calls' plain forms on a small cache."""
    n_pages, layers, nkv, hd = 8300, 32, 8, 128                    # 4.35e9 keys
    small_k, small_v = br.pool(12, layers, nkv, hd, 5)
    far = torch.tensor([8299, 8210, 8193, 8298, 8250, 8201, 8297, 8222, 4097, 8290, 2, 8233])      # page i of the small cache lies here
    k = torch.empty(n_pages, layers, nkv, 16, hd, dtype=torch.bfloat16, device="cuda")
    v = torch.empty(n_pages, layers, nkv, hd, 16, dtype=torch.bfloat16, device="cuda")
    assert k.numel() > 2 ** 32

    def put():
        k[far.cuda()], v[far.cuda()] = small_k.cuda(), small_v.cuda()

    def same():
        return torch.equal(k[far.cuda()].cpu(), small_k) and torch.equal(v[far.cuda()].cpu(), small_v)

    put()
    i32 = dict(dtype=torch.int32)
    near = torch.tensor([[0, 3, 6, 9], [1, 2, 4, 10]], **i32)
    table = far[near.long()].to(torch.int32)
    lens, nodes, mask = torch.tensor([41, 17], **i32), torch.tensor([9, 5], **i32), br.random_masks(2, 9, 3)
    q = torch.randn(2, 9, 32, hd, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16)
    ref, mass, dots = br.tree_attention_ref(q, small_k, small_v, layers, near, lens, nodes, mask)
    bound = br.tree_attention_bound(ref, mass, dots, hd, 64)
    wide = torch.full((2, 4096), 0x7ffffff0, **i32)
    wide[:, :4] = table
    for t in (table, wide):
        got = dl.tree_attention(q.cuda(), k, v, layers, t.cuda(), lens.cuda(), nodes.cuda(), mask.cuda()).cpu().double()
        live = ~ref.isnan()
        assert ((got - ref).abs() <= bound)[live].all()
    # in place (few pages), and from one row's pages into others
    pos = torch.tensor([[43, 45, 46], [18, 20, 21]], **i32)
    table_d = table.cuda()
    dl.kv_compact(k, v, table_d, pos.cuda(), torch.tensor([3, 2], **i32).cuda(), table_d, lens.cuda())
    br.compact_ref(small_k, small_v, near, pos, torch.tensor([3, 2], **i32), near, lens)
    assert same()
    src = torch.tensor([[i for i in range(0, 41, 2)] + [0] * 60], **i32)
    out_near = torch.tensor([[11, 8, 7, 5, 5, 5]], **i32)
    out_near[0, 4:] = -1
    dl.kv_compact(k, v, table_d[:1], src.cuda(), torch.tensor([21], **i32).cuda(), torch.where(out_near >= 0, far[out_near.long()].to(torch.int32), out_near).cuda(),
                  torch.tensor([16], **i32).cuda())
    br.compact_ref(small_k, small_v, near[:1], src, torch.tensor([21], **i32), out_near, torch.tensor([16], **i32))
    assert same()
    # a fork copies a part-filled page between far pages
    new, new_lens, counts = torch.full((3, 5), -1, **i32).cuda(), torch.zeros(3, **i32).cuda(), torch.zeros(2, **i32).cuda()
    dl.kv_fork(k, v, table_d, lens.cuda(), torch.tensor([1, 0, 0], **i32).cuda(), far[[11, 8]].to(torch.int32).cuda(), torch.tensor([2], **i32).cuda(), new, new_lens, counts)
    assert new[2].tolist() == [8299, 8298, 8233, -1, -1] and counts.tolist() == [0, 0]
    small_k[11], small_v[11] = small_k[6], small_v[6]
    assert same()


# ---------------------------------------------------------------- streams, graphs, several calls at once
def test_calls_on_streams_and_in_graphs():
    """Each operator captured twice into graphs that are replayed interleaved, on changed inputs, beside an eager call on a third stream."""
    torch.manual_seed(0)
    q, k, v, table, lens, nodes, m = [dev(t) for t in make_tree(8, 2, 128, [300, 77], [9, 9], 9, seed=31)]
    logits, scores = torch.randn(2, 4, 5000, device="cuda"), torch.zeros(2, 4, device="cuda")
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs, graphs = [], []
    for s in streams:
        o = torch.zeros_like(q)
        b = [torch.zeros(2, 4, dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32)]
        with torch.cuda.stream(s):                               # loads the kernels before the capture
            dl.tree_attention(q, k, v, 2, table, lens, nodes, m, out=o)
            dl.beam_select(logits, scores, *b)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            dl.tree_attention(q, k, v, 2, table, lens, nodes, m, out=o)
            dl.beam_select(logits, scores, *b)
        outs.append((o, b))
        graphs.append(graph)
    for turn in range(3):
        q.copy_(torch.randn_like(q, dtype=torch.float32))
        logits.normal_()
        lens.copy_(torch.tensor([300 - 100 * turn, 77], dtype=torch.int32))
        torch.cuda.synchronize()
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        third = torch.cuda.Stream()
        eager = torch.zeros_like(q)
        third.wait_stream(torch.cuda.current_stream())
        dl.tree_attention(q, k, v, 2, table, lens, nodes, m, out=eager, stream=third)
        torch.cuda.synchronize()
        want = br.beam_ref(logits.cpu(), scores.cpu(), 4)
        for o, b in outs:
            assert torch.equal(o, eager)
            assert np.array_equal(b[1].cpu().numpy(), want[1]) and np.array_equal(b[2].cpu().numpy(), want[2])


def test_what_a_call_makes_belongs_to_its_stream():
    """A call on another stream than the busy current one: its output is not cleared by work of the current stream that comes late,
    and its workspace is no memory that the current stream still reads."""
    q, k, v, table, lens, nodes, m = [dev(t) for t in make_tree(4, 2, 64, [100], [5], 5, seed=8)]
    logits, scores = torch.randn(1, 4, 5000, device="cuda"), torch.zeros(1, 4, device="cuda")
    outs, want = [[torch.zeros(1, 4, dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32)] for _ in range(2)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):                                 # loads the kernels
        att = dl.tree_attention(q, k, v, 1, table, lens, nodes, m)
        dl.beam_select(logits, scores, *want)
    torch.cuda.synchronize()
    shape = dl.BeamC(*(dict(batch=1, beams=4, vocab=5000, k=4, dtype=0, row_stride=5000).get(n, 0) for n, _ in dl.BeamC._fields_))
    n = dl.load_library().del_beam_workspace_bytes(dl.C.byref(shape))
    held = torch.full((n,), 77, dtype=torch.uint8, device="cuda")
    seen = torch.zeros_like(held)
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)                                # the current stream is busy for some 50 ms
    seen.copy_(held)
    del held
    got = dl.tree_attention(q, k, v, 1, table, lens, nodes, m, stream=side)
    dl.beam_select(logits, scores, *outs, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, att)
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    assert (seen == 77).all()


@pytest.mark.parametrize("vocab,beams", [(700, 4), (40000, 12)])      # selection in one launch, in two
def test_calls_in_a_row_are_calls_one_by_one(vocab, beams):
    """Steps of selection, fork, compaction and attention that feed one another without a wait on the host, and replayed from a graph,
    give what they give when the host waits after each call: no kernel reads before the one before it has written."""
    nh, nkv, hd, cols, steps, n_pages = 8, 2, 64, 12, 10, 400
    i32 = dict(dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(beams)
    k0, v0 = br.pool(n_pages, 3, nkv, hd, 2, "cuda")
    logits = [torch.randn(1, beams, vocab, generator=g).cuda() for _ in range(steps)]
    q = [torch.randn(beams, 3, nh, hd, generator=g).to(torch.bfloat16).cuda() for _ in range(steps)]
    order = torch.randperm(n_pages, generator=g).to(torch.int32)
    keep = (1 + 2 * torch.arange(60)).to(torch.int32).repeat(beams, 1).cuda()
    n_keep, zero, page_ids = torch.full((beams,), 40, **i32), torch.zeros(beams, **i32), order[:beams * 8].view(beams, 8).contiguous().cuda()
    other = order[beams * 8: beams * 11].view(beams, 3).contiguous().cuda()
    spare = order[beams * 11:].cuda()
    spares, n_spare = [spare[i * beams:(i + 1) * beams] for i in range(steps)], torch.tensor([beams], **i32)

    class State:
        def __init__(self):
            self.k, self.v = k0.clone(), v0.clone()
            self.tables = [torch.zeros(beams, cols, **i32) for _ in range(steps + 1)]
            self.tables[0][:, :8] = page_ids
            self.lens = [torch.full((beams,), 97, **i32) if i == 0 else torch.zeros(beams, **i32) for i in range(steps + 1)]
            self.scores = [torch.zeros(1, beams, device="cuda") for _ in range(steps + 1)]
            self.tokens, self.rows = ([torch.zeros(1, beams, **i32) for _ in range(steps)] for _ in range(2))
            self.counts = [torch.zeros(2, **i32) for _ in range(steps)]
            self.out = [torch.zeros_like(x) for x in q]

        def run(self, wait):
            for i in range(steps):
                for call in (lambda: dl.beam_select(logits[i], self.scores[i], self.scores[i + 1], self.tokens[i], self.rows[i]),
                             lambda: dl.kv_fork(self.k, self.v, self.tables[i], self.lens[i], self.rows[i].view(-1), spares[i], n_spare, self.tables[i + 1],
                                                self.lens[i + 1], self.counts[i], room=3),
                             lambda: dl.kv_compact(self.k, self.v, self.tables[i + 1], keep, n_keep, other, zero),
                             lambda: dl.tree_attention(q[i], self.k, self.v, 1 + i % 3, self.tables[i + 1], self.lens[i + 1], out=self.out[i]),
                             lambda: dl.kv_compact(self.k, self.v, self.tables[i + 1], keep[:, 30:35], n_keep, self.tables[i + 1], self.lens[i + 1])):
                    call()
                    if wait:
                        torch.cuda.synchronize()

        def all(self):
            return [self.k, self.v, *self.tables[1:], *self.lens[1:], *self.scores[1:], *self.tokens, *self.rows, *self.counts, *self.out]

    one, row, graphed = State(), State(), State()
    torch.cuda.synchronize()
    one.run(True)
    row.run(False)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.run(False)
    graph.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(one.all(), row.all(), graphed.all()):
        assert torch.equal(a, b) and torch.equal(a, c)
    assert not torch.equal(one.k, k0)


def test_beam_search_over_shared_pages():
    """The operators as they are used together: beams that share pages are attended one token at a time, selected and forked; every
    step against the dense form over each beam's own history."""
    torch.manual_seed(4)
    batch, beams, nh, nkv, hd, vocab, steps, prompt = 3, 4, 4, 2, 64, 500, 20, 21
    rows, cols, i32 = batch * beams, 6, dict(dtype=torch.int32, device="cuda")
    n_pages = rows * cols + 8
    emb_k, emb_v, emb_q = (torch.randn(vocab, n, hd).to(torch.bfloat16) for n in (nkv, nkv, nh))
    head = (torch.randn(vocab, nh * hd) * 0.3).to(torch.bfloat16)
    k, v = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((n_pages, 1, nkv, 16, hd), (n_pages, 1, nkv, hd, 16)))
    history = [[int(t) for t in torch.randint(0, vocab, (prompt,))] for _ in range(batch)]
    tables, lens = [torch.full((rows, cols), -1, **i32) for _ in range(2)], [torch.zeros(rows, **i32) for _ in range(2)]
    free, counts = [torch.zeros(n_pages, **i32) for _ in range(2)], [torch.zeros(2, **i32) for _ in range(2)]
    free[0].copy_(torch.randperm(n_pages))
    counts[0][0] = n_pages
    # the prompts: one old row per item without positions, forked with room for the prompt into the first beam alone
    first = torch.tensor([b // beams if b % beams == 0 else -1 for b in range(rows)], **i32)
    dl.kv_fork(k, v, torch.zeros(batch, cols, **i32), torch.zeros(batch, **i32), first, free[0], counts[0], tables[1], lens[1], counts[1], room=prompt, free_pages=free[1])
    cur = 1

    def write(row, pos, tok):
        pg = int(tables[cur][row, pos // 16])
        k[pg, 0, :, pos % 16] = emb_k[tok].cuda()
        v[pg, 0, :, :, pos % 16] = emb_v[tok].cuda()

    for item in range(batch):
        for p, t in enumerate(history[item]):
            write(item * beams, p, t)
        lens[cur][item * beams] = prompt - 1                      # the last token is the node that is attended
    seqs = [history[r // beams][:] for r in range(rows)]
    scores = torch.full((batch, beams), float("-inf"), device="cuda")
    scores[:, 0] = 0.0
    finished = torch.zeros(batch, beams, dtype=torch.bool, device="cuda")
    outs = [torch.zeros(batch, beams, dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32)]
    reordered = 0
    for step in range(steps):
        # attention of the last token (it lies in the cache), logits, selection, fork with room for the next token
        q = torch.stack([emb_q[s[-1]] for s in seqs]).cuda()[:, None].contiguous()
        att = dl.tree_attention(q, k, v, 1, tables[cur], lens[cur])
        att[scores.view(-1) == float("-inf")] = 0                 # rows without a history yet (their lens are 0: they see one empty slot)
        logits = (att.float().view(rows, -1) @ head.float().cuda().T).view(batch, beams, vocab)
        dl.beam_select(logits, scores, *outs, finished=finished, eos=1)
        want = br.beam_ref(logits.cpu(), scores.cpu(), beams, finished.cpu(), 1)
        assert np.array_equal(outs[1].cpu().numpy(), want[1]) and np.array_equal(outs[2].cpu().numpy(), want[2])
        # the attention against the dense form of the beam's own history
        for r in range(rows):
            if float(scores.view(-1)[r]) == float("-inf"):
                continue
            K, V = emb_k[seqs[r]].double(), emb_v[seqs[r]].double()
            for h in range(nh):
                w = torch.softmax(K[:, h // 2] @ emb_q[seqs[r][-1], h].double() * hd ** -0.5, 0)
                mass = (w[:, None] * V[:, h // 2].abs()).sum(0)
                ref = (w[:, None] * V[:, h // 2]).sum(0)
                assert ((att[r, 0, h].cpu().double() - ref).abs() <= 2.0 ** -8 * (1.05 * mass + ref.abs())).all()
        parents, tokens = outs[2].view(-1).cpu().tolist(), outs[1].view(-1).cpu().tolist()
        reordered += parents != list(range(rows))
        lens[cur] += 1
        dl.kv_fork(k, v, tables[cur], lens[cur], outs[2].view(-1), free[cur], counts[cur], tables[1 - cur], lens[1 - cur], counts[1 - cur],
                   room=1, free_pages=free[1 - cur])
        cur = 1 - cur
        assert int(counts[cur][1]) == 0
        seqs = [seqs[p] + [t] for p, t in zip(parents, tokens)]
        for r in range(rows):
            assert int(lens[cur][r]) == len(seqs[r]) - 1
            write(r, len(seqs[r]) - 1, seqs[r][-1])
        scores.copy_(outs[0])
        finished.copy_(outs[1] == 1)
    assert reordered > 3
