"""Histories that share pages, move and change their cache: each attends as one that was written by itself does, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2511_14881_amd.history import HistoryStore

pytestmark = pytest.mark.gpu
HEADS, D = 2, 128


def rows(gen, n, heads=HEADS):
    return torch.randn((n, heads, D), generator=gen, device="cuda").to(torch.bfloat16)


def attend(store, users, q):
    return store.attend(users, q, [q.shape[0] // len(users)] * len(users))


def test_forked_moved_and_resized_histories_attend_as_their_own_do():
    gen = torch.Generator(device="cuda").manual_seed(5)
    k, v, more_k, more_v = (rows(gen, n) for n in (530, 530, 300, 300))
    q = rows(gen, 6, 4 * HEADS)
    store, alone = HistoryStore(4, 40, HEADS, D, 14), HistoryStore(4, 40, HEADS, D, 14)
    store.append([0, 1], k, v, [330, 200])
    store.mass[0] = 2.0
    store.fork([0, 1], [2, 3])
    assert len(store.free) == 40 - 6 - 4 and (store.mass[2] == 2.0).all()
    alone.append([0, 1], k, v, [330, 200])
    alone.append([2, 3], k, v, [330, 200])
    assert torch.equal(attend(store, [0, 1, 2], q), attend(alone, [0, 1, 2], q))
    # the forks go on by themselves, with events of other sizes: scales of the shared pages would change
    for s in (store, alone):
        s.append([2, 0, 3], 5.0 * more_k[:171], more_v[:171], [100, 1, 70])
    assert torch.equal(attend(store, [0, 1, 2, 3], q[:4]), attend(alone, [0, 1, 2, 3], q[:4]))
    assert len(set(store.tables[0, :5]) & set(store.tables[2, :5])) == 5 and store.tables[0, 5] != store.tables[2, 5]
    want = attend(store, [0, 2, 3], q)
    store.release([1])
    moved = store.compact()
    assert moved > 0 and store.tables.max() == (store.shares > 0).sum() - 1 and torch.equal(attend(store, [0, 2, 3], q), want)
    for n in ((store.shares > 0).sum(), 64):
        store.resize(int(n))
        assert store.cache.n_pages == n and torch.equal(attend(store, [0, 2, 3], q), want)
    for s in (store, alone):
        s.append([0, 2], more_k[171:], more_v[171:], [64, 65])
    assert torch.equal(attend(store, [0, 2, 3], q), attend(alone, [0, 2, 3], q))


def test_many_forks_of_one_history():
    """As candidates for what follows an event: 30 continuations of one history, each with an event of its own."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    k, v, new_k, new_v = (rows(gen, n) for n in (1000, 1000, 31, 31))
    store = HistoryStore(31, 16 + 30, HEADS, D, 17)  # the last page 31 times: one history keeps it
    store.append([0], k, v, [1000])
    store.fork([0] * 30, range(1, 31))
    store.append(range(31), new_k, new_v)
    assert len(store.free) == 0 and store.shares.max() == 31 and (store.shares == 1).sum() == 31
    q = rows(gen, 31, HEADS)
    out = attend(store, range(31), q)
    for u in (0, 1, 30):
        one = HistoryStore(1, 16, HEADS, D, 16)
        one.append([0], k, v, [1000])
        one.append([0], new_k[u:u + 1], new_v[u:u + 1])
        plain = attend(one, [0], q[u:u + 1])
        # another number of histories may be split otherwise: on both sides one rounding to bf16, weights rounded to 11 bits beside another
        # maximum, and 1001 / 16 + 64 roundings of sums in fp32
        top = max(v.float().abs().max(), new_v.float().abs().max())
        bound = 2 * (2.0 ** -8 * plain.float().abs() + (2.0 ** -12 + (1001 / 16 + 64) * 2.0 ** -23) * top)
        assert ((out[u].float() - plain[0].float()).abs() <= bound[0]).all()
    assert store.release(range(1, 31)) == 30 and store.compact() >= 0
    assert np.array_equal(np.sort(store.tables[0, :16]), np.arange(16))
