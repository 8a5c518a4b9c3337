"""Searches and their helpers on a stream other than the current one: what a call allocates for itself is not handed out before the call has run."""
import numpy as np
import pytest
import torch

from paper_2511_14881_amd import binding as st
from paper_2511_14881_amd import synth
from tests.test_gpu_kv_streams import busy, note

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def index():
    w = synth.make_workload(synth.CONFIGS["tiny"], device="cuda")
    bloom = st.st_bloom_build(w.feat_offsets, w.feat_ids, w.cfg.n_items, w.cfg.m_bits, w.cfg.k_hashes)
    yield w, bloom
    bloom.free()


def call_of(name, w, bloom):
    n_q, K = len(w.filt_offsets) - 1, w.cfg.top_k
    items = bloom, w.items, w.item_scale
    ids = np.asarray(w.filt_ids)[np.minimum(np.asarray(w.filt_offsets)[:-1], len(w.filt_ids) - 1)]
    program = np.full(n_q, st.ST_OP_LEAF, np.int32), ids, np.arange(n_q + 1)
    if name == "search":
        return lambda **kw: st.st_search(*items, w.queries, w.query_scale, w.filt_ids, w.filt_offsets, K, **kw)
    if name == "multitask":
        q, s = w.queries[:, None].repeat(1, 2, 1), w.query_scale.repeat_interleave(2)
        return lambda **kw: st.st_search_multitask(*items, q, s, [0.5, 2.0], w.filt_ids, w.filt_offsets, K, **kw)
    if name == "expr":
        return lambda **kw: st.st_search_expr(*items, w.queries, w.query_scale, *program, K, **kw)
    table = w.items.float() * w.item_scale[:, None]
    return lambda **kw: st.st_quantize_global(table, **kw)


@pytest.mark.parametrize("name", ["search", "multitask", "expr", "quantize"])
def test_memory_of_a_call_on_another_stream_is_not_handed_out_before_it_ran(name, index, monkeypatch):
    call = call_of(name, *index)
    want = [x.clone() for x in call()]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    side = torch.cuda.Stream()
    kept = busy(side)
    asked, sizes, empty = [], [], torch.empty

    def watched(*a, **kw):
        t = note(asked, empty(*a, **kw))
        sizes.append(t.numel() * t.element_size())
        return t

    monkeypatch.setattr(torch, "empty", watched)
    got = call(stream=side)
    monkeypatch.undo()
    assert asked and not side.query()  # the call has memory of its own and is still to run
    now = [torch.empty(size, dtype=torch.uint8, device="cuda") for size in sizes]
    assert not {t.data_ptr() for t in now} & set(asked)
    for t in now:
        t.fill_(0xFF)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    del kept


def test_masks_on_another_stream_are_not_cleared_from_the_current_one(index):
    """The current stream is busy when the call is made: a clearing queued there would come after the mask."""
    w, bloom = index
    n_q = len(w.filt_offsets) - 1
    ids = np.asarray(w.filt_ids)[np.minimum(np.asarray(w.filt_offsets)[:-1], len(w.filt_ids) - 1)]
    calls = [lambda **kw: st.st_bloom_mask(bloom, w.filt_ids, w.filt_offsets, **kw),
             lambda **kw: st.st_bloom_mask_expr(bloom, np.full(n_q, st.ST_OP_LEAF, np.int32), ids, np.arange(n_q + 1), **kw)]
    for call in calls:
        want = call()
        assert want.any()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        kept = busy(torch.cuda.current_stream())
        got = call(stream=side)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        del kept
