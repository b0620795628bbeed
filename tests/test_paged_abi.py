"""CPU: what the operators on device buffers refuse, before anything reaches a GPU, and the page addressing by its formula."""
import numpy as np
import pytest

import paper_2407_19947_amd as pkg
from operators_util import key_at, value_at, keep_reference, sample_reference

P = 1 << 20                        # an aligned address nobody reads: the calls are refused


def cache(**kw):
    return pkg.StairsPagedCache(**dict(dict(k=P, v=P, dtype=pkg.DTYPE_BF16, n_pages=8, page_size=64, n_kv_heads=4, head_dim=128), **kw))


def plan(**kw):
    return pkg.StairsPagePlan(**dict(dict(n_seqs=2, max_blocks=4, n_pages=8, page_size=64, max_rows=16, cached=P, fresh=P, held=P, n_free=P,
                                          block_table=P, free_pages=P, held_out=P, n_free_out=P, row_start=P, seq_len=P, position=P, slot=P), **kw))


def rows(**kw):
    return pkg.StairsPagedRows(**dict(dict(rows=3, n_heads=8, q=P, k=P, v=P, q_out=P, q_stride=1024, k_stride=512, v_stride=512, q_out_stride=1024,
                                           position=P, slot=P, rope_theta=1e4), **kw))


def attn(**kw):
    return pkg.StairsPagedAttention(**dict(dict(n_seqs=2, max_blocks=4, rows=4, n_heads=8, max_fresh=2, q=P, out=2 * P, q_stride=1024, out_stride=1024,
                                                block_table=P, row_start=P, seq_len=P, scale=0.0, workspace=P, workspace_bytes=1 << 40), **kw))


def sampling(**kw):
    return pkg.StairsSampling(**dict(dict(dtype=pkg.DTYPE_FP32, rows=2, vocab=100, ld=100, logits=P, uniform=P, token=P), **kw))


def refused(call, code=-1):
    with pytest.raises(pkg.StairsError) as e:
        call()
    assert e.value.code == code


@pytest.mark.parametrize("bad", [dict(n_seqs=-1), dict(n_seqs=1025), dict(max_blocks=0), dict(n_pages=0), dict(page_size=16), dict(page_size=96),
                                 dict(max_rows=-1), dict(cached=None), dict(fresh=None), dict(held=None), dict(n_free=None), dict(block_table=None),
                                 dict(free_pages=None), dict(held_out=None), dict(n_free_out=None), dict(row_start=None), dict(seq_len=None),
                                 dict(position=None), dict(slot=None), dict(n_pages=1 << 26, page_size=32), dict(max_blocks=1 << 24, page_size=128)])
def test_plan_refuses(bad):
    refused(lambda: pkg.stairs_paged_plan(plan(**bad)))


CACHES = [dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 2), dict(dtype=pkg.DTYPE_FP32), dict(dtype=9), dict(n_pages=0), dict(page_size=0),
          dict(page_size=48), dict(page_size=512), dict(n_kv_heads=0), dict(head_dim=32), dict(head_dim=96), dict(n_pages=1 << 25)]


@pytest.mark.parametrize("bad", CACHES)
def test_a_pool_that_is_none_is_refused(bad):
    refused(lambda: pkg.stairs_paged_append(cache(**bad), rows()))
    refused(lambda: pkg.stairs_paged_attention(cache(**bad), attn()))
    refused(lambda: pkg.stairs_paged_attention_workspace(cache(**bad), attn()))


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(n_heads=-1), dict(q=None), dict(k=None), dict(v=None), dict(q_out=None), dict(slot=None),
                                 dict(position=None), dict(q=P + 2), dict(k=P + 4), dict(v=P + 8), dict(q_out=P + 2), dict(q_stride=1016),
                                 dict(q_stride=1028), dict(k_stride=500), dict(k_stride=516), dict(v_stride=0), dict(v_stride=-512), dict(q_out_stride=8),
                                 dict(rope_theta=-1.0), dict(rope_theta=float("nan")), dict(rope_theta=float("inf")), dict(q_stride=1032)])
def test_append_refuses(bad):
    refused(lambda: pkg.stairs_paged_append(cache(), rows(**bad)))


@pytest.mark.parametrize("bad", [dict(n_seqs=-1), dict(n_seqs=1025), dict(max_blocks=0), dict(rows=-1), dict(n_heads=6), dict(n_heads=0), dict(max_fresh=-1),
                                 dict(q=None), dict(out=None), dict(out=P), dict(block_table=None), dict(row_start=None), dict(seq_len=None),
                                 dict(q=P + 8), dict(out=2 * P + 2), dict(q_stride=1000), dict(out_stride=1025), dict(scale=float("nan")),
                                 dict(scale=float("inf")), dict(max_blocks=1 << 25), dict(rows=1 << 25)])
def test_attention_refuses(bad):
    refused(lambda: pkg.stairs_paged_attention(cache(), attn(**bad)))


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(rows=-1), dict(rows=(1 << 21) + 1), dict(vocab=0), dict(vocab=524289, ld=524289), dict(ld=99), dict(logits=None),
                                 dict(token=None), dict(logits=P + 2), dict(dtype=pkg.DTYPE_FP16, logits=P + 1)])
def test_sampling_refuses(bad):
    refused(lambda: pkg.stairs_sample_device(sampling(**bad)))


def test_attention_refuses_more_work_groups_than_a_launch_has():
    many = dict(n_heads=4096, q_stride=4096 * 64, out_stride=4096 * 64, max_fresh=1)
    heads = cache(n_kv_heads=4096, head_dim=64)
    assert pkg.stairs_paged_attention_workspace(heads, attn(rows=4000, **many)) > 0
    refused(lambda: pkg.stairs_paged_attention_workspace(heads, attn(rows=1 << 20, **many)))
    refused(lambda: pkg.stairs_paged_attention(heads, attn(rows=1 << 20, **many)))


@pytest.mark.parametrize("n", [(1 << 29) - 31, 1 << 30, 2 ** 31 - 1])
def test_append_refuses_more_work_groups_than_a_launch_has(n):
    refused(lambda: pkg.stairs_paged_append(cache(), rows(rows=n)))


def test_a_workspace_does_not_shrink_with_the_call():
    sizes = [pkg.stairs_paged_attention_workspace(cache(), attn(n_seqs=n, rows=r)) for n, r in ((1, 2), (2, 4), (1024, 2048))]
    assert sizes == sorted(sizes)


def test_nothing_to_do_is_no_error():
    pkg.stairs_paged_append(cache(), rows(rows=0))
    pkg.stairs_paged_attention(cache(), attn(n_seqs=0))
    pkg.stairs_paged_attention(cache(), attn(rows=0))
    pkg.stairs_sample_device(sampling(rows=0))


def test_null_arguments():
    L = pkg.lib()
    assert L.stairs_paged_plan(None, None) == -1
    assert L.stairs_paged_append(None, None, None) == -1
    assert L.stairs_paged_attention(cache(), None, None) == -1
    assert L.stairs_paged_attention_workspace(None, attn()) == -1
    assert L.stairs_sample_device(None, None) == -1
    assert L.stairs_sample_workspace(None) == -1
    assert L.stairs_set_truncation(None, 0, 1.0, 0.0) == -1


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("ps", [32, 64, 256])
def test_every_element_of_a_page_has_a_place_of_its_own(ps, hd):
    p, e = np.meshgrid(np.arange(ps), np.arange(hd), indexing="ij")
    for at in (key_at, value_at):
        assert np.array_equal(np.sort(at(p, e, hd).ravel()), np.arange(ps * hd))


def test_the_sampling_reference_by_hand():
    x = np.log([4.0, 1.0, 2.0, 2.0, 1.0])
    assert keep_reference(x, top_k=3)[0].tolist() == [True, False, True, True, False]
    assert keep_reference(x, top_k=2)[0].tolist() == [True, False, True, False, False]        # equal logits by index
    # (4 of 10 in front of the next; 0.4 as a float is a little more than that)
    assert keep_reference(x, top_p=0.4)[0].tolist() == [True, False, True, False, False]
    assert keep_reference(x, top_p=0.399)[0].tolist() == [True, False, False, False, False]
    assert keep_reference(x, top_p=0.41)[0].tolist() == [True, False, True, False, False]
    assert keep_reference(x, min_p=0.5)[0].tolist() == [True, False, True, True, False]
    assert keep_reference(x, top_k=3, top_p=0.5)[0].tolist() == [True, False, False, False, False]   # 4 of 8
    assert [sample_reference(x, u)[0] for u in (0.0, 0.39, 0.41, 0.51, 0.71, 0.95)] == [0, 0, 1, 2, 3, 4]
    assert sample_reference(x, 0.5, temperature=0)[0] == 0
    assert sample_reference(np.full(3, -np.inf), 0.5)[0] == -1
