"""Pages that histories of a store share, give back and move, on the host.  The kernels are stubs: a page is a number that an append
changes and a copy takes over, so that each history's pages can be followed.  None of it touches a GPU."""
import types

import numpy as np
import pytest
import torch

from paper_2511_14881_amd import binding as st
from paper_2511_14881_amd.history import HistoryStore
from tests.test_history_host import D, HEADS, rows


@pytest.fixture
def store(monkeypatch):
    class Batch(types.SimpleNamespace):
        def __init__(self, tables, lengths, n_tok, offsets=None, max_tok=None, max_len=None):
            super().__init__(tables=tables.numpy().copy(), lengths=lengths.numpy().copy(), n_tok=n_tok, max_tok=max_tok,
                             offsets=None if offsets is None else offsets.numpy())

    def empty(pages, heads, d):
        return types.SimpleNamespace(n_pages=pages, n_heads=heads, d=d, held=[()] * pages)  # a page: the events written to it

    def append(cache, batch, k, v):
        counts = np.full(len(batch.lengths), batch.max_tok) if batch.offsets is None else np.diff(batch.offsets)
        wrote = []
        for table, length, n in zip(batch.tables, batch.lengths, counts):
            touched = set()
            for t in range(length - n, length):
                page = table[t // 64]
                if t % 64 == 0:
                    cache.held[page] = ()
                assert len(cache.held[page]) == t % 64
                cache.held[page] += (next(events),)
                touched.add(page)
            wrote += touched
        assert len(set(wrote)) == len(wrote)  # no page is written by two histories

    def copy(a, b, src, dst):
        src, dst = src.tolist(), dst.tolist()
        assert len(set(dst)) == len(dst) and not (a is b and set(src) & set(dst))
        for i, j in zip(src, dst):
            b.held[j] = a.held[i]
        copies.append(len(src))

    def evict(batch, mass, budget, sink=0, recent=1):
        from tests import kv_reference as R
        return tuple(torch.from_numpy(x) for x in R.evict(batch.tables, batch.lengths.tolist(), mass.numpy(), budget, sink, recent))

    events, copies = iter(range(1 << 30)), []
    monkeypatch.setattr(torch.Tensor, "cuda", lambda self: self)
    monkeypatch.setattr(st, "KvBatch", Batch)
    monkeypatch.setattr(st.KvCache, "empty", empty)
    zeros = torch.zeros
    monkeypatch.setattr(torch, "zeros", lambda *a, device=None, **kw: zeros(*a, **kw))
    for name, call in (("append", append), ("copy", copy), ("evict", evict)):
        monkeypatch.setattr(st, "st_kv_" + name, call)
    made = HistoryStore(5, 20, HEADS, D, 6)
    made.copies = copies
    return made


def history(store, user):
    held = []
    for b in range(-(-store.lengths[user] // 64)):
        held += store.cache.held[store.tables[user, b]]
    assert len(held) == store.lengths[user]
    return held


def append(store, users, counts):
    store.append(users, rows(sum(counts)), rows(sum(counts)), counts)


def consistent(store):
    n = store.cache.n_pages
    used = store.tables[store.tables >= 0]
    assert np.array_equal(np.bincount(used, minlength=n), store.shares) and len(store.shares) == n
    assert sorted(store.free) == np.flatnonzero(store.shares == 0).tolist()
    assert np.array_equal((store.tables >= 0).sum(1), -(-store.lengths // 64))
    return True


def test_a_fork_shares_pages_until_one_of_the_histories_grows(store):
    append(store, [0, 1], [130, 64])
    store.mass[0] = 3.0
    store.fork([0, 0, 1], [2, 3, 4])
    assert consistent(store) and len(store.free) == 20 - 4 and not store.copies
    assert history(store, 2) == history(store, 0) and store.lengths.tolist() == [130, 64, 130, 130, 64]
    assert (store.mass[2] == 3.0).all() and (store.mass[4] == 0.0).all()
    before = history(store, 0)
    # three histories share a page with two events: two of them get copies, the third keeps it; user 4's pages are full
    append(store, [0, 2, 3, 4], [1, 2, 3, 1])
    assert consistent(store) and store.copies == [2]
    assert [history(store, u)[:130] == before for u in (0, 2, 3)] == [True] * 3
    assert len({store.tables[u, 2] for u in (0, 2, 3)}) == 3 and store.tables[0, 0] == store.tables[3, 0]
    assert store.tables[4, 0] == store.tables[1, 0] and store.tables[4, 1] >= 0 > store.tables[1, 1]
    assert len(set(history(store, 0)) & set(history(store, 2))) == 130


def test_pages_come_free_with_the_last_history(store):
    append(store, [0], [200])
    store.fork([0], [1])
    append(store, [1], [1])
    assert len(store.free) == 20 - 5
    assert store.release([0]) == 1 and store.lengths[0] == 0 and consistent(store)  # the page that user 1 has a copy of
    assert len(history(store, 1)) == 201
    store.fork([1], [0])
    assert store.evict([0, 1], 2, recent=1) == 2 and consistent(store)
    assert store.release([1, 0]) == 2 and len(store.free) == 20 and consistent(store)
    assert store.release([]) == 0


def test_forks_that_are_refused_change_nothing(store):
    append(store, [0, 1], [10, 10])
    for users, to in (([0], [1]), ([0, 1], [2]), ([0, 1], [2, 2]), ([5], [2]), ([0], [-1]), ([0], [0])):
        with pytest.raises(ValueError):
            store.fork(users, to)
    assert consistent(store) and store.lengths.tolist() == [10, 10, 0, 0, 0]
    store.fork([], [])
    store.fork([2], [3])  # an empty history
    assert store.lengths.tolist() == [10, 10, 0, 0, 0] and consistent(store)
    # no page is left for the copy
    append(store, [2, 3, 4], [384, 384, 384])
    with pytest.raises(ValueError, match="free"):
        append(store, [0], [64])
    store.release([4])
    store.fork([0], [4])
    store.release([1])
    append(store, [1], [384])
    before = store.tables.copy(), store.shares.copy(), list(store.free)
    assert len(store.free) == 1
    with pytest.raises(ValueError, match="2 pages are needed"):
        append(store, [0], [60])
    assert np.array_equal(before[0], store.tables) and np.array_equal(before[1], store.shares) and before[2] == store.free


def test_pages_move_to_the_front_and_into_another_cache(store):
    append(store, [0, 1, 2], [130, 300, 64])
    store.fork([1], [3])
    store.release([0])
    held = {u: history(store, u) for u in (1, 2, 3)}
    assert store.compact() == 3 and consistent(store)
    assert sorted(set(store.tables[store.tables >= 0].tolist())) == list(range(6))
    assert {u: history(store, u) for u in (1, 2, 3)} == held and store.compact() == 0
    with pytest.raises(ValueError, match="in use"):
        store.resize(5)
    for n in (6, 31, 9):
        store.resize(n)
        assert store.cache.n_pages == n and consistent(store) and {u: history(store, u) for u in (1, 2, 3)} == held
    append(store, [3, 0], [1, 20])
    assert consistent(store) and history(store, 3)[:300] == held[3]


def test_histories_follow_plain_lists(store):
    rng = np.random.default_rng(3)
    plain = [[] for _ in range(5)]
    for step in range(300):
        what = rng.choice(["append", "append", "append", "fork", "release", "compact", "resize"])
        users = rng.permutation(5)[: rng.integers(1, 4)]
        try:
            if what == "append":
                counts = rng.integers(0, 90, len(users))
                append(store, users, counts.tolist())
                for u, n in zip(users, counts):
                    now = history(store, u)
                    assert now[: len(now) - n] == plain[u]
                    plain[u] = now
            elif what == "fork" and len(users) > 1:
                store.fork(users[:1], users[1:2])
                plain[users[1]] = list(plain[users[0]])
            elif what == "release":
                store.release(users[:1])
                plain[users[0]] = []
            elif what == "compact":
                store.compact()
            elif what == "resize":
                store.resize(int(rng.integers(8, 25)))
        except ValueError:
            pass
        assert consistent(store) and [history(store, u) for u in range(5)] == plain
