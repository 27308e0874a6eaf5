"""The tcgen05 form of the tree attention: one CTA's blocks of keys in every number, over values that come late; calls in a row, in graphs
and on several streams; whole models whose tree rounds take it."""
import pytest
import torch

import branch_ref as br
import paper_2504_05598_b200 as dl
from test_gpu_branching import check_tree_once, make_tree

pytestmark = pytest.mark.gpu

# heads whose tiles of 16 rows do not fit the device at once: these calls take the tcgen05 form, one tile per CTA, whatever their length
ONE_TILE = [(40, 40, 128, 64, 1), (40, 40, 64, 64, 2)]            # query heads, kv heads, head dimension, nodes, sequences


@pytest.mark.parametrize("nh,nkv,hd,n,batch", ONE_TILE)
@pytest.mark.parametrize("length", [40, 130, 300, 420, 700])
def test_one_tile_waits_for_all_of_its_products(nh, nkv, hd, n, batch, length):
    """max_len = 1 gives all blocks of a sequence to one CTA: 1 to 6 of them.  Nothing is in L2 when a call begins and every value
    page lies megabytes from the next, so that products wait for their values; each call gives the same bits, and those are right."""
    lens = [length, max(0, length - 128)][:batch]
    q, k, v, table, lens, nodes, m = make_tree(nh, nkv, hd, lens, [n] * batch, n, seed=length, layers=1)
    want = check_tree_once(q, k, v, 1, table, lens, nodes, m, max_len=1)
    spread = 64                                                   # pages of a pool in which only every 64th is in use
    n_pages = k.shape[0]
    far_k, far_v = (torch.zeros(n_pages * spread, *t.shape[1:], dtype=torch.bfloat16, device="cuda") for t in (k, v))
    far_k[::spread], far_v[::spread] = k.cuda(), v.cuda()
    far = torch.where(table < n_pages, table * spread, table).cuda()
    q, lens, nodes, m = q.cuda(), lens.cuda(), nodes.cuda(), m.cuda()
    flush = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    outs = [torch.zeros_like(q) for _ in range(20)]
    for out in outs:
        flush.zero_()
        dl.tree_attention(q, far_k, far_v, 1, far, lens, nodes, m, out=out, max_len=1)
    torch.cuda.synchronize()
    for out in outs:
        assert torch.equal(out, want)


@pytest.mark.parametrize("nh,nkv,hd,n", [(4, 2, 64, 3), (40, 40, 128, 64)])
def test_the_error_word_reaches_the_kernel(monkeypatch, nh, nkv, hd, n):
    """A caller's word stays as it was where no wait runs out; it is the one the library is given; what is no such word is refused."""
    q, k, v, table, lens, nodes, m = (t.cuda() for t in make_tree(nh, nkv, hd, [50], [n], n))
    word = torch.tensor([0, 5, 0], dtype=torch.int32, device="cuda")
    want = dl.tree_attention(q, k, v, 1, table, lens, nodes, m)
    assert torch.equal(dl.tree_attention(q, k, v, 1, table, lens, nodes, m, error=word[1:2]), want)
    assert word.tolist() == [0, 5, 0]
    for bad in (word, word[1:2].float(), word[1:2].cpu(), word[:0]):
        with pytest.raises(dl.DelError) as e:
            dl.tree_attention(q, k, v, 1, table, lens, nodes, m, error=bad)
        assert e.value.code == dl.EINVAL
    given = []

    class Library:
        @staticmethod
        def del_tree_attention(kv, args, stream):
            given.append(dl.TreeAttnC.from_buffer_copy(args).error)
            return dl.OK

    monkeypatch.setattr(dl, "_lib", Library)
    dl.tree_attention(q, k, v, 1, table, lens, nodes, m, error=word[1:2])
    dl.tree_attention(q, k, v, 1, table, lens, nodes, m)
    assert given == [word[1:2].data_ptr(), None]


def shape_of(tiles):
    """(sequences, nodes, columns of the tables) with 8 query and 2 kv heads of dimension 128 that take the tcgen05 form, one tile of rows
    per CTA or two."""
    return {1: (4, 20, 128), 2: (40, 40, 128)}[tiles]


@pytest.mark.parametrize("tiles", [1, 2])
def test_calls_in_a_row_are_calls_one_by_one(tiles):
    """Attention whose output is the next one's query, a small call of the mma.sync form between, an accepted path moved together in place and
    a fork that changes tables, without a wait on the host and replayed from a graph: the same bits as with a wait after each call."""
    batch, n, cols = shape_of(tiles)
    nh, nkv, hd, steps = 8, 2, 128, 8
    i32, g = dict(dtype=torch.int32, device="cuda"), torch.Generator().manual_seed(tiles)
    held = 12                                                     # pages of a row at the start
    n_pages = batch * (held + 3 * steps)
    k0, v0 = br.pool(n_pages, 2, nkv, hd, 3, "cuda")
    order = torch.randperm(n_pages, generator=g).to(torch.int32).cuda()
    first = torch.zeros(batch, cols, **i32)
    first[:, :held] = order[: batch * held].view(batch, held)
    spares, n_spare = order[batch * held:].view(steps, -1), torch.tensor([3 * batch], **i32)
    start = torch.randint(20, 150, (batch,), generator=g).to(torch.int32).cuda()
    q0 = (3 * torch.randn(batch, n, nh, hd, generator=g)).to(torch.bfloat16).cuda()
    nodes = torch.randint(n // 2, n + 1, (batch,), generator=g).to(torch.int32).cuda()
    masks = br.random_masks(batch, n, 5).cuda()
    path = torch.tensor([0, 2, 3, 7], **i32)
    n_path = torch.full((batch,), 4, **i32)
    parents = [torch.randint(0, batch, (batch,), generator=g).to(torch.int32).cuda() for _ in range(steps)]

    class State:
        def __init__(self):
            self.k, self.v = k0.clone(), v0.clone()
            self.tables = [first.clone()] + [torch.zeros(batch, cols, **i32) for _ in range(steps)]
            self.lens = [start.clone()] + [torch.zeros(batch, **i32) for _ in range(steps)]
            self.src = [torch.zeros(batch, 4, **i32) for _ in range(steps)]
            self.counts = [torch.zeros(2, **i32) for _ in range(steps)]
            self.q = [q0.clone()] + [torch.zeros_like(q0) for _ in range(steps)]
            self.low = [torch.zeros_like(q0) for _ in range(steps)]
            self.small = [torch.zeros(batch, 1, nh, hd, dtype=torch.bfloat16, device="cuda") for _ in range(steps)]
            self.error = torch.zeros(1, **i32)

        def run(self, wait):
            for i in range(steps):
                for call in (lambda: dl.tree_attention(self.q[i], self.k, self.v, 1 + i % 2, self.tables[i], self.lens[i], nodes, masks, out=self.q[i + 1],
                                                       out_lo=self.low[i], scale=0.5, error=self.error),
                             lambda: dl.tree_attention(self.q[i + 1][:, :1], self.k, self.v, 1, self.tables[i], self.lens[i], out=self.small[i], max_len=300),
                             lambda: torch.add(self.lens[i][:, None], path, out=self.src[i]),
                             lambda: dl.kv_compact(self.k, self.v, self.tables[i], self.src[i], n_path, self.tables[i], self.lens[i]),
                             lambda: dl.kv_fork(self.k, self.v, self.tables[i], self.lens[i], parents[i], spares[i], n_spare, self.tables[i + 1], self.lens[i + 1],
                                                self.counts[i], room=n),
                             lambda: self.q[i + 1].mul_(4.0)):
                    call()
                    if wait:
                        torch.cuda.synchronize()

        def all(self):
            return [self.k, self.v, *self.tables, *self.lens, *self.counts, *self.q, *self.low, *self.small]

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
    assert not one.q[steps].isnan().any() and not torch.equal(one.k, k0)
    for a, b, c in zip(one.all(), row.all(), graphed.all()):
        assert torch.equal(a, b) and torch.equal(a, c)
    assert int(one.error) == int(row.error) == int(graphed.error) == 0
    ref = State()                                                 # the first step is right
    dl.tree_attention(q0, ref.k, ref.v, 1, first, start, nodes, masks, out=ref.q[1], out_lo=ref.low[0], scale=0.5)
    want, mass, dots = br.tree_attention_ref(q0[:2], k0, v0, 1, first[:2], start[:2], nodes[:2], masks[:2], 0.5)
    live = ~want.isnan()
    got = ref.q[1][:2].cpu().double() + ref.low[0][:2].cpu().double()
    assert ((got - want).abs() <= br.tree_attention_bound(want, mass, dots, hd, 200, low=True))[live].all()
    assert torch.equal(ref.low[0], one.low[0])


@pytest.mark.parametrize("tiles", [1, 2])
def test_calls_on_streams_and_in_graphs(tiles):
    """Two graphs replayed side by side on changed inputs, beside an eager call on a third stream; all use the device's tensor memory."""
    batch, n, cols = shape_of(tiles)
    q, k, v, table, lens, nodes, m = (t.cuda() for t in make_tree(8, 2, 128, [100 + 37 * (b % 4) for b in range(batch)], [n] * batch, n, seed=31, cols=cols))
    streams, outs, graphs = [torch.cuda.Stream() for _ in range(2)], [], []
    for s in streams:
        o = torch.zeros_like(q)
        with torch.cuda.stream(s):                               # loads the kernel before the capture
            dl.tree_attention(q, k, v, 2, table, lens, nodes, m, out=o)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            for _ in range(3):
                dl.tree_attention(q, k, v, 2, table, lens, nodes, m, out=o)
        outs.append(o)
        graphs.append(graph)
    for turn in range(4):
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(turn)))
        lens.copy_(torch.tensor([100 + 37 * (b % 4) - 20 * turn for b in range(batch)], dtype=torch.int32))
        torch.cuda.synchronize()
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        third, eager = torch.cuda.Stream(), torch.zeros_like(q)
        third.wait_stream(torch.cuda.current_stream())
        dl.tree_attention(q, k, v, 2, table, lens, nodes, m, out=eager, stream=third)
        torch.cuda.synchronize()
        alone = dl.tree_attention(q, k, v, 2, table, lens, nodes, m)
        for o in outs + [eager]:
            assert torch.equal(o, alone)
