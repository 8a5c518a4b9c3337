"""Refusals of the entry points on cached histories, and their workspaces: none of it touches a GPU (the pointers
are numbers that are never followed)."""
import ctypes as C

import pytest

from paper_2511_14881_amd import binding as st

P = 1 << 20  # an aligned address


def cache(**kw):
    c = st._KvCacheC(P, P, P, P, P, 100, 4, 128)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def batch(**kw):
    b = st._KvBatchC(P, P, None, 2, 50, 6, 3, 3000)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def ref(x):
    return None if x is None else C.cast(C.pointer(x), C.c_void_p)


def attend(c, b, **kw):
    a = dict(q=P, stride=8 * 128, dtype=0, heads=8, scale=0.1, causal=1, mask=None, words=0, blocks=None, n_sel=0, out=P,
             lse=None, mass_in=None, decay=1.0, mass_out=None, ws=P, nbytes=1 << 40)
    a.update(kw)
    return st.lib().st_kv_attend(ref(c), ref(b), *a.values(), None)


def select(c, b, **kw):
    a = dict(q=P, stride=8 * 128, dtype=0, heads=8, causal=1, mask=None, words=0, n_sel=8, sink=1, recent=1, out=P, ws=P,
             nbytes=1 << 40)
    a.update(kw)
    return st.lib().st_kv_select(ref(c), ref(b), *a.values(), None)


def append(c, b, **kw):
    a = dict(k=P, ks=512, v=P, vs=512, dtype=0)
    a.update(kw)
    return st.lib().st_kv_append(ref(c), ref(b), *a.values(), None)


def evict(b, **kw):
    a = dict(mass=P, heads=4, budget=10, sink=1, recent=2, t=P, n=P, m=P, f=P, nf=P)
    a.update(kw)
    return st.lib().st_kv_evict(ref(b), *a.values(), None)


BAD_CACHE = [dict(d=100), dict(d=0), dict(d=32), dict(n_heads=0), dict(n_heads=1025), dict(n_pages=0), dict(n_pages=1 << 31),
             dict(k=P + 8), dict(bounds=None), dict(k_scale=None)]
BAD_BATCH = [dict(n_seq=-1), dict(max_blocks=0), dict(max_blocks=16385), dict(max_len=3201), dict(max_len=-1), dict(max_tok=7),
             dict(n_tok=7), dict(n_tok=-1), dict(tables=None), dict(lengths=None), dict(n_seq=0)]


@pytest.mark.parametrize("call", [attend, select, append])
def test_bad_caches_and_batches_are_refused(call):
    for kw in BAD_CACHE:
        assert call(cache(**kw), batch()) == st.ST_EINVAL, kw
        assert st.last_error()
    for kw in BAD_BATCH:
        assert call(cache(), batch(**kw)) == st.ST_EINVAL, kw
    assert call(None, batch()) == st.ST_EINVAL and call(cache(), None) == st.ST_EINVAL


def test_bad_calls_are_refused():
    nan = float("nan")
    for kw in (dict(q=None), dict(q=P + 2), dict(stride=1020), dict(stride=1016), dict(dtype=2), dict(heads=6), dict(heads=3),
               dict(heads=0), dict(scale=nan), dict(scale=float("inf")), dict(decay=nan), dict(mask=P, words=46), dict(mask=P + 4, words=50),
               dict(blocks=P), dict(blocks=P, n_sel=16385), dict(n_sel=4), dict(out=None), dict(out=P + 8), dict(mass_in=P),
               dict(ws=P + 128)):
        assert attend(cache(), batch(), **kw) == st.ST_EINVAL, kw
    for kw in (dict(q=None), dict(heads=5), dict(n_sel=0), dict(n_sel=16385), dict(sink=-1), dict(recent=-1), dict(sink=7, recent=2),
               dict(out=None), dict(ws=P + 64), dict(mask=P, words=0)):
        assert select(cache(), batch(), **kw) == st.ST_EINVAL, kw
    for kw in (dict(k=None), dict(v=None), dict(ks=508), dict(vs=504), dict(dtype=-1)):
        assert append(cache(), batch(), **kw) == st.ST_EINVAL, kw
    for kw in (dict(heads=0), dict(recent=0), dict(sink=-1), dict(budget=2), dict(mass=None), dict(t=None), dict(nf=None)):
        assert evict(batch(), **kw) == st.ST_EINVAL, kw
    for kw in BAD_BATCH[:-1]:
        assert evict(batch(**kw)) == st.ST_EINVAL, kw
    read = st.lib().st_kv_read
    assert read(ref(cache()), ref(batch()), 0, P, P, P, None) == st.ST_EINVAL
    assert read(ref(cache()), ref(batch()), 1, P + 4, P, P, None) == st.ST_EINVAL
    assert read(ref(cache(v=None)), ref(batch()), 1, P, P, P, None) == st.ST_EINVAL


def test_workspaces():
    L = st.lib()
    size = L.st_kv_attend_workspace_bytes
    b, c = batch(), cache()
    plain, mass = size(ref(c), ref(b), 8, 0, 0), size(ref(c), ref(b), 8, 0, 1)
    assert 256 <= plain < mass and plain % 256 == 0 and mass % 256 == 0
    assert mass - plain >= 6 * 8 * 47 * 8  # a pair to each row and block
    assert attend(c, b, mass_out=P, nbytes=mass - 256) == st.ST_EWORKSPACE
    assert attend(c, b, mass_out=P, ws=None) == st.ST_EWORKSPACE
    need = L.st_kv_select_workspace_bytes(ref(c), ref(b), 8, 8)
    assert need >= 6 * 4 * 47 * 4
    assert select(c, b, nbytes=need - 1) == st.ST_EWORKSPACE
    for bad in (lambda: size(ref(c), ref(b), 7, 0, 0), lambda: size(None, ref(b), 8, 0, 0), lambda: size(ref(c), ref(b), 8, -1, 0),
                lambda: L.st_kv_select_workspace_bytes(ref(c), ref(b), 8, 0), lambda: size(ref(cache(d=48)), ref(b), 8, 0, 0)):
        assert bad() == st.ST_EINVAL


def test_slot_order_of_values():
    from tests.kv_reference import SLOTS
    assert sorted(SLOTS) == list(range(64)) and SLOTS[:5].tolist() == [0, 1, 2, 3, 16] and SLOTS[16] == 4 and SLOTS[32] == 8
