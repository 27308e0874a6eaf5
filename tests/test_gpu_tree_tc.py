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
