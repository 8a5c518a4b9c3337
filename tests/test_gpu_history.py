"""The store of histories: what it hands out, attends to and takes back, against the plain implementation, and the
serving loop as a command."""
import json
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2511_14881_amd import binding as st
from paper_2511_14881_amd.history import HistoryStore
from tests import kv_reference as R
from tests.test_gpu_kv import check_out, queries

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Mirror(R.Host):
    """The plain side of a store: pages as the store deals them out."""

    def __init__(self, store):
        n, h, b, d = store.cache.k.shape
        self.heads, self.d, self.max_blocks = h, d, store.max_blocks
        self.k, self.v = np.zeros((n, h, b, d), np.int8), np.zeros((n, h, b, d), np.int8)
        self.ks, self.vs = np.zeros((n, h), np.float32), np.zeros((n, h), np.float32)
        self.bounds = np.zeros((n, h, 2, d), np.int8)

    def follow(self, store, users):
        self.tables, self.lens = store.tables[users], store.lengths[users].tolist()
        return self


def test_store_follows_plain_through_appends_and_evictions():
    rng = np.random.default_rng(1)
    store = HistoryStore(4, 24, 2, 64, 8)
    plain = Mirror(store)
    mass = np.zeros((4, 2, 8))
    for step, (users, counts) in enumerate([([0, 1, 2], [130, 64, 1]), ([3, 1], [200, 70]), ([0, 1, 2, 3], [1, 1, 1, 1]), ([2], [90]),
                                            ([0, 3], [60, 100])]):
        users = np.array(users)
        k, v = queries(rng, sum(counts), 2, 64, "bf16"), queries(rng, sum(counts), 2, 64, "bf16")
        store.append(users, k.cuda(), v.cuda(), counts)
        R.append(plain.follow(store, users), k, v, np.concatenate([[0], np.cumsum(counts)]).tolist())
        everyone = np.flatnonzero(store.lengths)
        q = queries(rng, len(everyone), 4, 64, "bf16")
        out = store.attend(everyone, q.cuda(), [1] * len(everyone), causal=True, track=True, decay=0.5)
        want, _, mass[everyone], reach = R.attend(plain.follow(store, everyone), q, 64 ** -0.5, True, mass=mass[everyone].astype(np.float32), decay=0.5)
        check_out(out, want, reach, plain, "bf16")
        assert np.allclose(store.mass.cpu().numpy(), mass, rtol=1e-4, atol=1e-5)
    before = store.tables.copy(), store.lengths.copy(), store.mass.cpu().numpy(), len(store.free)
    freed = store.evict([0, 1, 3], 2, sink=0, recent=1)
    want = R.evict(before[0][[0, 1, 3]], before[1][[0, 1, 3]], before[2][[0, 1, 3]], 2, 0, 1)
    assert freed == want[4].sum() and len(store.free) == before[3] + freed
    assert np.array_equal(store.tables[[0, 1, 3]], want[0]) and np.array_equal(store.lengths[[0, 1, 3]], want[1])
    assert np.array_equal(store.tables[2], before[0][2])
    in_use = store.tables[store.tables >= 0].tolist()
    assert sorted(in_use + store.free) == list(range(24))
    q = queries(rng, 12, 4, 64, "bf16")
    out = store.attend([0, 1, 2, 3], q.cuda(), [3, 3, 3, 3], n_sel=1)
    plain.follow(store, [0, 1, 2, 3])
    want, _, _, reach = R.attend(plain, q, 64 ** -0.5, False, blocks=R.select(plain, q, 1, False, 0, 0))
    check_out(out, want, reach, plain, "bf16")


def test_store_refuses_what_does_not_fit():
    store = HistoryStore(2, 3, 1, 64, 2)
    rows = torch.zeros((129, 1, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="blocks"):
        store.append([0], rows, rows, [129])
    store.append([0], rows[:128], rows[:128], [128])
    with pytest.raises(ValueError, match="pages"):
        store.append([1], rows[:65], rows[:65], [65])
    assert store.lengths.tolist() == [128, 0] and len(store.free) == 1


def test_serving_loop_runs():
    run = subprocess.run([sys.executable, "-m", "paper_2511_14881_amd.history", "--items", "20000", "--users", "5", "--events", "700",
                          "--candidates", "20", "--select", "3", "--budget", "8", "--steps", "4"], cwd=ROOT, capture_output=True,
                         text=True, timeout=100)
    assert run.returncode == 0, run.stderr[-2000:]
    said = json.loads(run.stdout.strip().splitlines()[-1])
    assert said["finite"] and said["pages_freed"] > 0 and said["longest"] <= 8 * st.ST_KV_BLOCK
