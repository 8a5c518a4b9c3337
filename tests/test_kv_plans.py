"""How the calls of tests/test_gpu_kv_paths.py would run, asked of the host part alone: each takes the path that it is there for, and together
they take every one."""
import ctypes as C

import numpy as np
import pytest

from paper_2511_14881_amd import binding as st
from tests.test_gpu_kv_paths import ATTEND, SELECT

P = 1 << 20  # an aligned address, never followed

# waves (0: the kernel for many rows), least number of blocks to a split, wavefronts of the join
RUNS = {
    "one wavefront": (1, 65, 0), "one wavefront, mask": (1, 65, 0), "one wavefront, all rows in a tile": (1, 11, 0),
    "one wavefront, d = 256": (1, 65, 0),
    "long splits": (4, 257, 0), "long splits, mask": (4, 257, 0), "long splits, d = 96": (4, 257, 0), "long splits, d = 256": (4, 257, 0),
    "few rows, d = 64": (4, 20, 1), "few rows, d = 96": (4, 20, 1), "few rows, d = 256": (4, 20, 1),
    "many rows": (0, 129, 0), "many rows, causal": (0, 129, 0), "many rows, mask": (0, 129, 0), "many rows, mask, d = 128": (0, 129, 0),
    "many rows, d = 256": (0, 129, 0), "many rows, mask, d = 256": (0, 129, 0), "many rows, few blocks to a workgroup": (0, 2, 4),
    "join, d = 64": (4, 4, 4), "join, d = 96": (4, 4, 4), "join, d = 256": (4, 4, 4), "join, many rows, d = 64": (0, 2, 4),
    "join, many rows, d = 256": (0, 2, 4),
}
# one kernel scores and chooses, workgroups and rounds of the scores, keys to a lane of the choice; waves, least blocks to a split and join of the attention
CHOICES = {
    "200 blocks": (0, 1, 1, 4, 4, 9, 0), "300 blocks": (0, 2, 1, 8, 4, 4, 1), "700 blocks": (0, 3, 1, 16, 4, 4, 1),
    "1500 blocks": (0, 6, 1, 0, 4, 4, 4), "3000 blocks": (0, 12, 1, 0, 4, 4, 4), "rounds": (0, 1, 3, 16, 4, 12, 0),
    "chunks and rounds": (0, 3, 2, 16, 4, 13, 1), "rounds, 1500 blocks": (0, 1, 6, 0, 4, 20, 1),
    "a token, 700 blocks": (1, 1, 1, 16, 4, 4, 1), "a token, 1024 blocks": (1, 1, 1, 16, 4, 4, 4), "a token, 1100 blocks": (1, 1, 1, 0, 4, 8, 1),
    "a token, 5000 blocks": (1, 1, 1, 0, 4, 100, 1), "a token, 5000 blocks, one sequence": (0, 20, 1, 0, 4, 4, 4),
    "a token, d = 256": (1, 1, 1, 16, 4, 4, 1), "a token, 16384 blocks": (0, 64, 1, 0, 4, 4, 4), "lookups": (0, 2, 1, 8, 1, 8, 0), "lookups, 70 blocks": (0, 1, 1, 4, 1, 70, 0),
    "lookups, d = 96": (0, 1, 1, 4, 1, 66, 0), "lookups, d = 256": (0, 1, 1, 4, 1, 6, 0), "270 of 300 blocks": (0, 2, 1, 8, 4, 257, 0),
}


def plan(d, heads, group, lens, n_q, n_sel=0, mass=0):
    top = max(lens)
    cache = st._KvCacheC(P, P, P, P, P, 1000, heads, d)
    batch = st._KvBatchC(P, P, None, len(lens), -(-top // 64), n_q * len(lens), n_q, top)
    out = np.zeros(10, np.int32)
    rc = st.lib().st_kv_host_plan(C.addressof(cache), C.addressof(batch), heads * group, n_sel, mass, out.ctypes.data)
    assert rc == st.ST_OK
    return dict(zip(("waves", "tiles", "chunk", "splits", "join_waves", "sum_lanes", "one", "chunks", "rounds", "keys"), out.tolist()))


def of_attend(name, mass=0):
    _, d, heads, group, lens, n_q, *_ = ATTEND[name]
    return plan(d, heads, group, lens, n_q, mass=mass)


def of_select(name, mass=0):
    _, d, heads, group, lens, n_q, _, _, n_sel, *_ = SELECT[name]
    return plan(d, heads, group, lens, n_q, n_sel, mass)


@pytest.mark.parametrize("name", list(ATTEND))
def test_attention_takes_the_path(name):
    got, (waves, chunk, join) = of_attend(name), RUNS[name]
    assert (got["waves"], got["join_waves"]) == (waves, join) and got["chunk"] >= chunk, got


@pytest.mark.parametrize("name", list(SELECT))
def test_selection_takes_the_path(name):
    got, want = of_select(name), CHOICES[name]
    assert tuple(got[k] for k in ("one", "chunks", "rounds", "keys", "waves")) == want[:5] and got["join_waves"] == want[6], got
    assert got["chunk"] >= want[5], got


def test_every_kernel_is_run_by_a_case():
    attend = {(ATTEND[n][1], of_attend(n)["waves"]) for n in ATTEND}
    assert attend >= {(d, w) for d in (64, 96, 128, 256) for w in (0, 1, 4)}
    selected = {(SELECT[n][1], of_select(n)["waves"]) for n in SELECT}
    assert selected >= {(d, w) for d in (64, 96, 128, 256) for w in (1, 4)}
    scores = {(SELECT[n][1], of_select(n)["one"]) for n in SELECT}
    assert scores >= {(d, one) for d in (64, 96, 128, 256) for one in (0, 1)}
    assert {of_select(n)["keys"] for n in SELECT if not of_select(n)["one"]} == {0, 4, 8, 16}
    assert {of_attend(n, mass=1)["sum_lanes"] for n in ATTEND} == {0, 16, 64}
    joins = {(ATTEND[n][1], of_attend(n)["join_waves"]) for n in ATTEND} | {(SELECT[n][1], of_select(n)["join_waves"]) for n in SELECT}
    assert joins >= {(d, w) for d in (64, 96, 256) for w in (1, 4)} | {(128, 1), (128, 4)}


def test_a_plan_is_refused_as_its_call_would_be():
    cache, batch = st._KvCacheC(P, P, P, P, P, 1000, 4, 128), st._KvBatchC(P, P, None, 2, 50, 6, 3, 3000)
    out = np.zeros(10, np.int32)

    def ask(c=cache, b=batch, heads=8, n_sel=0, to=out.ctypes.data):
        return st.lib().st_kv_host_plan(C.addressof(c), C.addressof(b), heads, n_sel, 0, to)

    assert ask() == st.ST_OK
    assert ask(to=None) == ask(heads=6) == ask(n_sel=-1) == ask(n_sel=16385) == st.ST_EINVAL
    assert ask(c=st._KvCacheC(P, P, P, P, P, 1000, 4, 100)) == ask(b=st._KvBatchC(P, P, None, 2, 50, 7, 3, 3000)) == st.ST_EINVAL
