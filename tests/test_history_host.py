"""What the store of histories does on the host: who gets which pages, and what it refuses.  The kernels are stubs and all
tensors lie in host memory, so none of it touches a GPU."""
import types

import numpy as np
import pytest
import torch

from paper_2511_14881_amd import binding as st
from paper_2511_14881_amd.history import HistoryStore

HEADS, D = 2, 64


@pytest.fixture
def calls(monkeypatch):
    """The kernel calls that were made, as (name, batch); a call named in `refuse` raises as a refused call does."""
    made, refuse = [], set()

    class Batch(types.SimpleNamespace):
        def __init__(self, tables, lengths, n_tok, offsets=None, max_tok=None, max_len=None):
            super().__init__(tables=tables, lengths=lengths, n_tok=n_tok, offsets=offsets, max_tok=max_tok, max_len=max_len)

    def call(name, result):
        def run(*args, **kw):
            batch = next(x for x in args if isinstance(x, Batch))
            if name in refuse:
                raise ValueError("k must be [n, heads, 64]")
            made.append((name, batch))
            return result(batch, *args, **kw)
        return run

    def evict(batch, *args, **kw):
        from tests import kv_reference as R
        _, mass, budget = args
        got = R.evict(batch.tables.numpy(), batch.lengths.tolist(), mass.numpy(), budget, kw["sink"], kw["recent"])
        return tuple(torch.from_numpy(x) for x in got)

    monkeypatch.setattr(torch.Tensor, "cuda", lambda self: self)
    monkeypatch.setattr(st, "KvBatch", Batch)
    monkeypatch.setattr(st.KvCache, "empty", lambda pages, heads, d: types.SimpleNamespace(n_pages=pages, n_heads=heads, d=d))
    zeros = torch.zeros
    monkeypatch.setattr(torch, "zeros", lambda *a, device=None, **kw: zeros(*a, **kw))
    monkeypatch.setattr(st, "st_kv_append", call("append", lambda *a, **kw: None))
    monkeypatch.setattr(st, "st_kv_attend", call("attend", lambda b, *a, **kw: torch.ones(b.n_tok)))
    monkeypatch.setattr(st, "st_kv_select", call("select", lambda b, *a, **kw: None))
    monkeypatch.setattr(st, "st_kv_evict", call("evict", evict))
    return types.SimpleNamespace(made=made, refuse=refuse)


def rows(n):
    return torch.zeros((n, HEADS, D), dtype=torch.bfloat16)


def state(store):
    return store.tables.copy(), store.lengths.copy(), list(store.free), store.mass.clone()


def same(a, b):
    return np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1]) and a[2] == b[2] and torch.equal(a[3], b[3])


def consistent(store):
    """Every page is free or one user's, and users have pages for what they hold."""
    used = store.tables[store.tables >= 0].tolist()
    held = -(-store.lengths // st.ST_KV_BLOCK)
    return sorted(used + store.free) == list(range(store.cache.n_pages)) and np.array_equal((store.tables >= 0).sum(1), held)


def test_appends_deal_pages_and_hand_the_kernel_lengths_after_them(calls):
    store = HistoryStore(3, 12, HEADS, D, 6)
    store.append([0, 2], rows(131), rows(131), [130, 1])
    store.append(np.array([2, 1]), rows(2), rows(2))
    assert store.lengths.tolist() == [130, 1, 2] and consistent(store)
    (_, first), (_, second) = calls.made
    assert first.lengths.tolist() == [130, 1] and first.offsets.tolist() == [0, 130, 131] and first.max_tok == 130 and first.max_len == 130
    assert second.lengths.tolist() == [2, 1] and second.offsets is None and second.max_tok == 1
    assert first.tables[:, 0].tolist() == store.tables[[0, 2], 0].tolist()


@pytest.mark.parametrize("users,counts", [([0, 0], [70, 3]), ([1, 0, 1], None)])
def test_a_user_named_twice_is_refused_where_a_history_would_be_written(calls, users, counts):
    store = HistoryStore(3, 12, HEADS, D, 6)
    store.append([0, 1], rows(200), rows(200), [100, 100])
    before = state(store)
    n = len(users) if counts is None else sum(counts)
    with pytest.raises(ValueError, match="twice"):
        store.append(users, rows(n), rows(n), counts)
    with pytest.raises(ValueError, match="twice"):
        store.evict(users, 1)
    with pytest.raises(ValueError, match="twice"):
        store.attend(users, rows(len(users)), [1] * len(users), track=True)
    assert same(before, state(store)) and consistent(store) and len(calls.made) == 1
    store.attend(users, rows(len(users)), [1] * len(users))  # two groups of one user's candidates: nothing is written
    assert calls.made[-1][1].tables[:, 0].tolist() == [store.tables[u, 0] for u in users]


@pytest.mark.parametrize("users", [[3], [-1], [0, 7], [[0, 1]], [0.5]])
def test_users_that_the_store_does_not_have_are_refused(calls, users):
    store = HistoryStore(3, 12, HEADS, D, 6)
    before = state(store)
    for call in (lambda: store.append(users, rows(2), rows(2), [1] * len(users)), lambda: store.evict(users, 1),
                 lambda: store.attend(users, rows(2), [1] * len(users))):
        with pytest.raises((ValueError, IndexError)):
            call()
    assert same(before, state(store)) and not calls.made


def test_a_refused_append_leaves_the_store_as_it_was(calls):
    store = HistoryStore(2, 4, HEADS, D, 3)
    store.append([0], rows(70), rows(70), [70])
    before = state(store)
    calls.refuse.add("append")
    for users, counts in (([0], [60]), ([1], [65]), ([0, 1], [1, 1])):
        with pytest.raises(ValueError):
            store.append(users, rows(3), rows(3), counts)
        assert same(before, state(store)) and consistent(store)
    calls.refuse.clear()
    for users, counts in (([0], [-1]), ([0, 1], [1]), ([0], [1, 2])):
        with pytest.raises(ValueError, match="counts"):
            store.append(users, rows(1), rows(1), counts)
        with pytest.raises(ValueError, match="counts"):
            store.attend(users, rows(1), counts)
    for users, counts in (([0], [200]), ([0, 1], [60, 190])):  # more blocks than a history has, more pages than are free
        with pytest.raises(ValueError, match="evict first"):
            store.append(users, rows(sum(counts)), rows(sum(counts)), counts)
    assert same(before, state(store)) and len(calls.made) == 1
    store.append([0, 1], rows(61), rows(61), [60, 1])
    assert store.lengths.tolist() == [130, 1] and consistent(store)


def test_pages_that_came_free_are_dealt_once(calls):
    rng = np.random.default_rng(0)
    store = HistoryStore(5, 40, HEADS, D, 9)
    for _ in range(60):
        users = rng.permutation(5)[: rng.integers(1, 6)]
        counts = rng.integers(0, 130, len(users))
        try:
            store.append(users, rows(int(counts.sum())), rows(int(counts.sum())), counts)
        except ValueError:
            store.evict(users, int(rng.integers(1, 4)))
        assert consistent(store)
    assert {"append", "evict"} <= {name for name, _ in calls.made}


def test_calls_of_no_users_do_nothing(calls):
    store = HistoryStore(2, 4, HEADS, D, 3)
    store.append([0], rows(5), rows(5), [5])
    before, made = state(store), len(calls.made)
    for none in ([], np.array([], np.int64), np.array([])):
        store.append(none, rows(0), rows(0))
        store.append(none, rows(0), rows(0), [])
        assert store.evict(none, 1) == 0
        out = store.attend(none, rows(0), [])
        assert out.shape == (0, HEADS, D) and out.dtype == torch.bfloat16
        assert store.attend(none, rows(0), [], n_sel=2, track=True).shape == (0, HEADS, D)
    assert same(before, state(store)) and len(calls.made) == made
