"""Operators of branching decoding: what their calls refuse, on the host (no kernel is launched here)."""
import ctypes as C

import pytest
import torch

import paper_2504_05598_b200 as dl

P = 1 << 20              # an aligned address that no refused call may touch


def kv(**over):
    d = dict(k_pages=P, v_pages=P, n_pages=8, n_layers=2, n_kv_heads=2, head_dim=64)
    d.update(over)
    return dl.Pages(*(d[n] for n, _ in dl.Pages._fields_))


def call(name, cls, good, over, pages=None):
    d = dict(good)
    d.update(over)
    a = cls(*(d[n] for n, _ in cls._fields_))
    lib = dl.load_library()
    if name == "del_beam_select":
        return lib.del_beam_select(C.byref(a), None)
    return getattr(lib, name)(C.byref(kv(**(pages or {}))), C.byref(a), None)


TREE = dict(q=P, out=P, out_lo=None, page_table=P, lens=P, nodes=None, mask=None, error=None, q_seq_stride=512, q_node_stride=256, out_seq_stride=512,
            out_node_stride=256, batch=1, max_nodes=2, n_heads=4, layer=1, table_cols=4, table_stride=4, max_len=0, scale=0.0)
COMPACT = dict(src_table=P, dst_table=P, src_pos=P, counts=P, dst_start=P, batch=1, max_count=4, src_cols=4, src_stride=4, dst_cols=4,
               dst_stride=4, pos_stride=4)
FORK = dict(table=P, lens=P, parents=P, spare=P, n_spare=P, new_table=2 * P, new_lens=2 * P, free_pages=None, counts=3 * P, n_old=2, n_new=2,
            old_cols=4, old_stride=4, new_cols=4, new_stride=4, spare_cap=4, room=1)
BEAM = dict(logits=P, scores=P, finished=None, out_scores=P, out_tokens=P, out_rows=P, workspace=P, workspace_bytes=1 << 20, row_stride=100, batch=2, beams=3, vocab=100, k=4, eos=0, dtype=0)

BAD_PAGES = [dict(k_pages=None), dict(v_pages=P + 8), dict(n_pages=0), dict(n_layers=0), dict(n_kv_heads=0), dict(head_dim=96)]


@pytest.mark.parametrize("over", [dict(q=None), dict(out=None), dict(page_table=None), dict(lens=None), dict(q=P + 2), dict(out=P + 8), dict(out_lo=P + 8),
                                  dict(lens=P + 2), dict(mask=P + 4), dict(q_node_stride=257), dict(out_seq_stride=4), dict(batch=0), dict(batch=65536),
                                  dict(max_nodes=0), dict(max_nodes=65), dict(n_heads=3), dict(n_heads=0), dict(n_heads=2050), dict(layer=0), dict(layer=3),
                                  dict(table_cols=0), dict(table_cols=1 << 28), dict(table_stride=-1), dict(max_len=-1), dict(scale=-1.0),
                                  dict(scale=float("nan")), dict(scale=float("inf"))])
def test_tree_attention_refuses(over):
    assert call("del_tree_attention", dl.TreeAttnC, TREE, over) == dl.EINVAL


@pytest.mark.parametrize("over", [dict(src_table=None), dict(dst_table=None), dict(src_pos=None), dict(counts=None), dict(dst_start=None),
                                  dict(src_pos=P + 1), dict(batch=0), dict(batch=65536), dict(max_count=0), dict(src_cols=0), dict(dst_cols=0),
                                  dict(src_stride=-1), dict(dst_stride=-4), dict(pos_stride=-1)])
def test_compact_refuses(over):
    assert call("del_kv_compact", dl.CompactC, COMPACT, over) == dl.EINVAL


@pytest.mark.parametrize("over", [dict(table=None), dict(lens=None), dict(parents=None), dict(spare=None), dict(n_spare=None), dict(new_table=None),
                                  dict(new_lens=None), dict(counts=None), dict(counts=3 * P + 2), dict(n_old=0), dict(n_old=1025), dict(n_new=0),
                                  dict(n_new=1025), dict(old_cols=0), dict(new_cols=0), dict(old_stride=3), dict(new_stride=3), dict(spare_cap=-1),
                                  dict(room=-1), dict(new_table=P), dict(new_table=P + 28), dict(new_lens=P + 4), dict(free_pages=P + 8),
                                  dict(counts=P)])
def test_fork_refuses(over):
    assert call("del_kv_fork", dl.ForkC, FORK, over) == dl.EINVAL


def test_fork_refuses_to_list_more_pages_than_it_can_mark():
    assert call("del_kv_fork", dl.ForkC, FORK, dict(free_pages=64 * P), dict(n_pages=(1 << 20) + 1)) == dl.EINVAL


@pytest.mark.parametrize("over", [dict(logits=None), dict(scores=None), dict(out_scores=None), dict(out_tokens=None), dict(out_rows=None), dict(logits=P + 2), dict(workspace=None), dict(workspace=P + 8),
                                  dict(batch=65536), dict(batch=2000, beams=64),
                                  dict(dtype=3), dict(dtype=-1), dict(batch=0), dict(beams=0), dict(beams=65), dict(vocab=0), dict(k=0), dict(k=65),
                                  dict(vocab=1, row_stride=1), dict(row_stride=99), dict(finished=P, eos=100), dict(finished=P, eos=-1)])
def test_beam_select_refuses(over):
    assert call("del_beam_select", dl.BeamC, BEAM, over) == dl.EINVAL


@pytest.mark.parametrize("over", BAD_PAGES)
def test_caches_that_are_refused(over):
    assert call("del_tree_attention", dl.TreeAttnC, TREE, {}, over) == dl.EINVAL
    assert call("del_kv_compact", dl.CompactC, COMPACT, {}, over) == dl.EINVAL
    assert call("del_kv_fork", dl.ForkC, FORK, {}, over) == dl.EINVAL


def test_sizes_that_counts_of_32_bits_do_not_hold():
    assert call("del_kv_compact", dl.CompactC, COMPACT, dict(max_count=(1 << 31) - 1, pos_stride=(1 << 31) - 1)) == dl.EINVAL
    far = dict(table=1 << 40, lens=1 << 41, new_table=1 << 42, new_lens=1 << 43)
    assert call("del_kv_fork", dl.ForkC, FORK, dict(far, n_new=1024, new_cols=1 << 21, new_stride=1 << 21, room=(1 << 31) - 1)) == dl.EINVAL


def test_null_structs():
    lib, pages = dl.load_library(), kv()
    for name in ("del_tree_attention", "del_kv_compact", "del_kv_fork"):
        assert getattr(lib, name)(C.byref(pages), None, None) == dl.EINVAL
        assert getattr(lib, name)(None, None, None) == dl.EINVAL
    assert lib.del_beam_select(None, None) == dl.EINVAL


def test_binding_refuses_host_tensors_and_wrong_types():
    k, v = torch.zeros(4, 1, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(4, 1, 2, 64, 16, dtype=torch.bfloat16)
    i = torch.zeros(1, 4, dtype=torch.int32)
    with pytest.raises(dl.DelError):
        dl.tree_attention(torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16), k, v, 1, i, i[0, :1])
    with pytest.raises(dl.DelError):
        dl.kv_compact(k, v, i, i, i[0, :1], i, i[0, :1])
    with pytest.raises(dl.DelError):
        dl.kv_fork(k.float(), v, i, i[0, :1], i[0, :1], i[0], i[0], i, i[0, :1], i[0, :2])
    with pytest.raises(dl.DelError):
        dl.beam_select(torch.zeros(1, 1, 8), torch.zeros(1, 1), torch.zeros(1, 2), i[:, :2], i[:, :2])


def test_context_calls_without_a_context():
    lib = dl.load_library()
    assert lib.del_verify_tree(None, 0, 0, None, None, None, None) == dl.EINVAL
    assert lib.del_fork(None, 0, 1, 1) == dl.EINVAL
