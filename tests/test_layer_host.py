"""Refusals and workspaces of the entry points of a layer around the cached histories: none of it touches a GPU (the pointers
are numbers that are never followed)."""
import ctypes as C

import numpy as np
import pytest

from paper_2511_14881_amd import binding as st

P = 1 << 20  # an aligned address
NAN = float("nan")


def norm(**kw):
    a = dict(x=P, xs=256, r=P, rs=256, w=P, dtype=0, n=5, d=256, normalise=1, eps=1e-6, total=P, ts=256, q=P, scale=P, y=None)
    a.update(kw)
    return st.lib().st_norm_rows(*a.values(), None)


def adapters(**kw):
    a = st._AdaptersC(P, P, P, 4, 16)
    for k, v in kw.items():
        setattr(a, k, v)
    return C.cast(C.pointer(a), C.c_void_p)


def project(ad=None, **kw):
    a = dict(x=P, xs=P, rows=20, k=128, w=P, ws=P, n=64, ad=ad, of=P if ad else None, dtype=0, out=2 * P, stride=64, work=P, nbytes=1 << 30)
    a.update(kw)
    return st.lib().st_project(*a.values(), None)


def rotate(sections=(16, 8, 8), **kw):
    a = dict(q=P, qs=512, qh=4, k=2 * P, ks=128, kh=1, d=128, dtype=0, n=9, positions=P, freqs=P,
             sections=np.asarray(sections, dtype=np.int32).ctypes.data_as(C.c_void_p), axes=len(sections), inter=0, inverse=0, oq=P,
             oqs=512, ok=2 * P, oks=128)
    a.update(kw)
    return st.lib().st_rotate(*a.values(), None)


def copy(from_c=None, to_c=None, **kw):
    c = [st._KvCacheC(P, P, P, P, P, 100, 4, 128) for _ in range(2)]
    for x, more in zip(c, (from_c or {}, to_c or {})):
        for k, v in more.items():
            setattr(x, k, v)
    a = dict(src=P, dst=P, n=3)
    a.update(kw)
    return st.lib().st_kv_copy(*(C.cast(C.pointer(x), C.c_void_p) for x in c), *a.values(), None)


def test_bad_norms_are_refused():
    for kw in (dict(dtype=3), dict(dtype=-1), dict(n=-1), dict(n=1 << 31), dict(d=0), dict(d=24), dict(d=16400), dict(eps=0.0), dict(eps=NAN),
               dict(eps=2.0), dict(eps=1e-13), dict(x=None), dict(q=None), dict(scale=None), dict(q=None, scale=None, total=None),
               dict(x=P + 8), dict(xs=255), dict(xs=250), dict(xs=252), dict(rs=248), dict(ts=260), dict(r=P + 2), dict(w=P + 4),
               dict(total=P + 8), dict(y=P + 2), dict(scale=P + 2), dict(ts=264, r=None), dict(x=P + 4096, ts=264)):
        assert norm(**kw) == st.ST_EINVAL, kw
        assert st.last_error()
    assert norm(n=(1 << 31) - 1, d=16384, xs=16384, rs=16384, ts=16384) == st.ST_EINVAL  # more workgroups than a launch has


def test_bad_projections_are_refused():
    ad = adapters()
    for kw in (dict(dtype=2), dict(rows=-1), dict(k=0), dict(k=24), dict(k=16400), dict(n=8), dict(n=72, stride=72), dict(n=65552, stride=65552),
               dict(x=None), dict(xs=None), dict(w=None), dict(ws=None), dict(out=None), dict(of=P), dict(x=P + 4), dict(w=P + 8),
               dict(ws=P + 4), dict(xs=P + 2), dict(out=P + 8), dict(stride=63), dict(stride=68), dict(stride=56)):
        assert project(**kw) == st.ST_EINVAL, kw
    for kw in (dict(of=None), dict(of=P + 2), dict(work=P + 128)):
        assert project(ad, **kw) == st.ST_EINVAL, kw
    for kw in (dict(a=None), dict(b=None), dict(alpha=None), dict(a=P + 8), dict(b=P + 2), dict(alpha=P + 1), dict(n_adapters=0),
               dict(n_adapters=65537), dict(rank=0), dict(rank=12), dict(rank=136)):
        assert project(adapters(**kw)) == st.ST_EINVAL, kw
    assert project(rows=(1 << 31) - 1, n=65536, stride=65536) == st.ST_EINVAL


def test_workspace_of_a_projection():
    size = st.lib().st_project_workspace_bytes
    assert size(20, 128, 64, None) == 256
    need = size(20, 128, 64, adapters())
    assert need >= 20 * 16 * 2 + 20 * 4 and need % 256 == 0
    assert project(adapters(), nbytes=need - 1) == st.ST_EWORKSPACE and project(adapters(), work=None) == st.ST_EWORKSPACE
    for args in ((-1, 128, 64, None), (1, 100, 64, None), (1, 128, 0, None), (1, 128, 64, adapters(rank=4))):
        assert size(*args) == st.ST_EINVAL


def test_bad_rotations_are_refused():
    for kw in (dict(dtype=2), dict(n=-1), dict(d=12), dict(d=520), dict(d=8), dict(qh=-1), dict(kh=-1), dict(kh=1025), dict(axes=0), dict(axes=9),
               dict(positions=None), dict(freqs=None), dict(q=None), dict(ok=None), dict(positions=P + 2),
               dict(freqs=P + 4), dict(qs=500), dict(qs=504), dict(oks=120), dict(q=P + 8), dict(oq=P + 2), dict(qs=520), dict(oks=136)):
        assert rotate(**kw) == st.ST_EINVAL, kw
    for sections in ((0,), (4,), (12,), (72,), (-8, 16), (64, 8), (1 << 30, 1 << 30, 1 << 30)):
        assert rotate(sections) == st.ST_EINVAL, sections


def test_bad_copies_are_refused():
    for kw in (dict(from_c=dict(d=100)), dict(to_c=dict(d=64)), dict(to_c=dict(n_heads=2)), dict(from_c=dict(k=None)), dict(to_c=dict(v=P + 8)),
               dict(to_c=dict(n_pages=0)), dict(n=-1), dict(src=None), dict(dst=None), dict(src=P + 2), dict(dst=P + 1), dict(n=(1 << 31) - 1)):
        assert copy(**kw) == st.ST_EINVAL, kw
    assert copy(n=0, src=None, dst=None) == st.ST_OK


def test_outputs_in_the_place_of_other_arrays_are_refused():
    """What a row's threads write may not be what another row's have yet to read."""
    q = P + (1 << 12)
    for kw in (dict(y=P), dict(y=q, r=q, total=None), dict(y=q, total=q), dict(x=q, ts=264, total=q), dict(r=q, ts=264, total=q)):
        assert norm(**kw) == st.ST_EINVAL, kw
    assert project(out=P) == st.ST_EINVAL and project(x=q, w=P, out=q) == st.ST_EINVAL
    apart = dict(q=P, k=2 * P, oq=q, ok=2 * q)
    for kw in (dict(oq=2 * P), dict(ok=P), dict(ok=q), dict(oq=2 * P, ok=P)):
        assert rotate(**{**apart, **kw}) == st.ST_EINVAL, kw


def test_calls_of_nothing_do_nothing():
    assert norm(n=0) == st.ST_OK and project(rows=0) == st.ST_OK and rotate(n=0) == st.ST_OK
    assert rotate(qh=0, kh=0, q=None, k=None, oq=None, ok=None) == st.ST_OK


def test_routes_of_projections():
    """Each of the ways a projection can run is taken by some call, and the sizes of the GPU tests take them all."""
    plan = st.st_project_host_plan
    assert plan(1, 512, 1024, 8, 16) == {"edge": 0, "inner_rows": 0, "order": 0}
    assert plan(1, 512, 1024) == {"edge": 0, "inner_rows": 0, "order": 0}
    assert plan(1, 4096, 1024, 8, 16) == {"edge": 0, "inner_rows": 1, "order": 0}
    assert plan(64, 512, 1024, 8, 16) == {"edge": 0, "inner_rows": 1, "order": 0}
    assert plan(384, 512, 1024, 8, 16) == {"edge": 0, "inner_rows": 1, "order": 0}
    assert plan(192, 512, 1024, 8, 128)["edge"] == 0 and plan(193, 512, 1024, 8, 128)["edge"] == 64
    assert plan(385, 512, 1024, 4, 16) == plan(65, 512, 8192 + 16, 4, 16) == {"edge": 64, "inner_rows": 16, "order": 0}
    assert plan(1001, 1040, 1296, 5, 8) == {"edge": 64, "inner_rows": 16, "order": 1}
    assert plan(16384, 4096, 5120, 16, 32) == {"edge": 256, "inner_rows": 32, "order": 1}
    assert plan(16384, 4096, 5120) == {"edge": 256, "inner_rows": 0, "order": 0}
    from tests.test_gpu_layer import LARGE, PROJECTIONS
    taken = [plan(rows, k, n, count, rank) for _, rows, k, n, count, rank, _ in LARGE + PROJECTIONS]
    assert {p["edge"] for p in taken} == {0, 64, 128, 256} and {p["inner_rows"] for p in taken} == {0, 1, 16, 32}
    assert {(p["edge"], p["order"]) for p in taken} >= {(64, 0), (64, 1), (128, 0), (128, 1), (256, 0), (256, 1)}
    for args in ((-1, 64, 64), (1, 60, 64), (1, 64, 60), (1, 64, 64, 1, 7)):
        with pytest.raises(st.StError):
            plan(*args)
