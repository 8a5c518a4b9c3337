"""The operators of a layer as they are used together: step by step against the plain implementations, each on what the step before
really gave; the loop as a command; captured graphs; and calls on another stream."""
import json
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2511_14881_amd import binding as st
from paper_2511_14881_amd.history import HistoryStore
from paper_2511_14881_amd.layer import HistoryLayer
from tests import layer_reference as R
from tests.test_gpu_kv_streams import busy, note

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def make(gen, dtype, heads=4, kv_heads=2, d=64, width=192, tenants=3, rank=16):
    def normal(*shape, size=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * size).to(dtype)

    def adapters(n, k):
        return normal(tenants, rank, k, size=k ** -0.5), normal(tenants, n, rank, size=0.2), torch.rand(tenants, generator=gen, device="cuda")

    n = (heads + 2 * kv_heads) * d
    freqs = torch.cat([10000.0 ** (-torch.arange(20) / 20), 1e-3 * 0.5 ** torch.arange(12)]).double().cuda()
    layer = HistoryLayer(heads, kv_heads, d, 1 + 0.1 * normal(width), normal(n, width, size=width ** -0.5), normal(width, heads * d, size=0.06),
                         (20, 12), freqs, adapters(n, width), adapters(width, heads * d))
    return layer, normal


def below(off, bound):
    assert (off <= bound).all(), f"{(off - bound).max()} over the bound"


def values(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_layer_is_its_steps_and_they_match_plain(dtype):
    gen = torch.Generator(device="cuda").manual_seed(3)
    layer, normal = make(gen, R.TYPES[dtype])
    store, other = (HistoryStore(3, 30, 2, 64, 10) for _ in range(2))
    counts = [70, 1, 130]
    tenants = torch.tensor([0] * 70 + [-1] + [2] * 130, dtype=torch.int32, device="cuda")
    x, residual = normal(201, 192), normal(201, 192)
    positions = torch.stack([torch.arange(201), 1_700_000_000 + 977 * torch.arange(201)]).int().cuda()
    out, total = layer(store, [0, 1, 2], x, positions, counts, tenants, residual)
    # by hand
    rows = st.st_norm_rows(x, layer.norm, residual, eps=layer.eps)
    h, q8, unit, rms, _ = R.norm(x.cpu(), layer.norm.cpu(), residual.cpu(), layer.eps, True)
    assert torch.equal(total, rows.total) and torch.equal(total.cpu(), h) and np.array_equal(rows.q.cpu().numpy(), q8)
    below(np.abs(values(rows.scale) - unit * rms), R.norm_bound(192) * unit * rms)
    qkv = st.st_project(rows.q, rows.scale, layer.qkv.w, layer.qkv.scale, layer.qkv.adapters, tenants)
    ad = layer.qkv.adapters
    want, bound = R.project(*(t.cpu() for t in (rows.q, rows.scale, layer.qkv.w, layer.qkv.scale, ad.a, ad.b, ad.alpha, tenants)), dtype=dtype)
    below(np.abs(values(qkv) - want), bound)
    heads = qkv.view(201, 8, 64)
    q, k = st.st_rotate(heads[:, :4], heads[:, 4:6], positions, layer.freqs, layer.sections)
    for got, part in ((q, heads[:, :4]), (k, heads[:, 4:6])):
        want, bound = R.rotate(part.cpu(), positions.cpu(), layer.freqs.cpu(), layer.sections, False, False, dtype)
        below(np.abs(values(got) - want), bound)
    other.append([0, 1, 2], k, heads[:, 6:], counts)
    assert all(torch.equal(getattr(store.cache, n)[store.tables[store.tables >= 0]], getattr(other.cache, n)[other.tables[other.tables >= 0]])
               for n in ("k_scale", "v_scale", "bounds"))
    seen = other.attend([0, 1, 2], q, counts, causal=True)
    rows = st.st_norm_rows(seen.view(201, 256), normalise=False)
    _, q8, unit, _, _ = R.norm(seen.view(201, 256).cpu(), None, None, 0.0, False)
    assert np.array_equal(rows.q.cpu().numpy(), q8) and np.array_equal(rows.scale.cpu().numpy(), unit.astype(np.float32))
    ad = layer.out.adapters
    again = st.st_project(rows.q, rows.scale, layer.out.w, layer.out.scale, ad, tenants)
    want, bound = R.project(*(t.cpu() for t in (rows.q, rows.scale, layer.out.w, layer.out.scale, ad.a, ad.b, ad.alpha, tenants)), dtype=dtype)
    below(np.abs(values(again) - want), bound)
    assert torch.equal(out, again)


def test_events_taken_in_at_once_or_one_by_one_and_candidates():
    gen = torch.Generator(device="cuda").manual_seed(4)
    layer, normal = make(gen, torch.bfloat16)
    x = normal(40, 192)
    positions = torch.stack([torch.arange(40), 100 * torch.arange(40)]).int().cuda()
    one, other = (HistoryStore(1, 4, 2, 64, 3) for _ in range(2))
    layer.take_in(one, [0], x, positions, [40])
    for t in range(40):
        out, _ = layer(other, [0], x[t:t + 1], positions[:, t:t + 1].contiguous())
    assert one.lengths[0] == other.lengths[0] == 40
    # a step is the block's scale at the end: half of one for the first rounding on each side, and half for each of the 39 events that may
    # have made the scale grow on the way, which rounds the older integers again
    batch = one.batch([0], [0])
    a, b = (st.st_kv_read(s.cache, s.batch([0], [0]), 1)[0] for s in (one, other))
    assert (a - b).abs().max() <= (1 + 39 / 2) * one.cache.k_scale.max()
    # candidates leave the histories as they are
    before = [t.clone() for t in (one.cache.k, one.cache.v, one.cache.k_scale)]
    rows = normal(9, 192)
    got, total = layer(one, [0], rows, positions[:, :9].contiguous(), [9], append=False, n_sel=1)
    assert got.shape == (9, 192) and total is rows and torch.isfinite(got.float()).all() and batch.n_tok == 0
    assert all(torch.equal(x, y) for x, y in zip(before, (one.cache.k, one.cache.v, one.cache.k_scale)))


def test_layer_refuses_weights_that_do_not_fit():
    w = torch.zeros((512, 64), dtype=torch.bfloat16, device="cuda")
    for heads, kv_heads, out in ((4, 3, 256), (4, 2, 128), (3, 2, 192), (0, 2, 0)):
        with pytest.raises(ValueError):
            HistoryLayer(heads, kv_heads, 64, w[0], w, torch.zeros((64, out), dtype=torch.bfloat16, device="cuda"), (8,), None)


def test_serving_loop_with_the_layer_runs():
    run = subprocess.run([sys.executable, "-m", "paper_2511_14881_amd.history", "--items", "20000", "--users", "5", "--events", "700",
                          "--candidates", "20", "--select", "3", "--budget", "8", "--steps", "4", "--layer"], cwd=ROOT, capture_output=True,
                         text=True, timeout=100)
    assert run.returncode == 0, run.stderr[-2000:]
    said = json.loads(run.stdout.strip().splitlines()[-1])
    assert said["finite"] and said["pages_freed"] > 0 and said["longest"] <= 8 * st.ST_KV_BLOCK and said["pages"] <= 5 * 8


def test_captured_steps_replay_as_they_run():
    """A decode step with all operators in one graph, and a second graph of the same operators on the same buffers; other inputs
    and eager work between the replays."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    layer, normal = make(gen, torch.bfloat16)
    n, old = 6, 200
    store = HistoryStore(n, n * 5, 2, 64, 5)
    store.append(range(n), normal(n * old, 2, 64), normal(n * old, 2, 64), [old] * n)
    store.append(range(n), normal(n, 2, 64), normal(n, 2, 64))  # pages for the token that each step writes
    batch = store.batch(np.arange(n), np.ones(n))
    x, residual = normal(n, 192), normal(n, 192)
    tenants = torch.tensor([0, 1, 2, 0, -1, 7], dtype=torch.int32, device="cuda")
    positions = torch.stack([torch.full((n,), old), torch.arange(n)]).int().cuda()
    rows, last = st.RowBuffers(n, 192, torch.bfloat16, total=True), st.RowBuffers(n, 192, torch.bfloat16, total=True)
    seen = st.RowBuffers(n, 256, torch.bfloat16)
    qkv = st.ProjectBuffers(n, 192, 512, torch.bfloat16, layer.qkv.adapters)
    back = st.ProjectBuffers(n, 256, 192, torch.bfloat16, layer.out.adapters)
    q0 = torch.empty((n, 4, 64), dtype=torch.bfloat16, device="cuda")
    attended = st.KvBuffers(store.cache, batch, q0)
    src, dst = torch.tensor([0, 1], dtype=torch.int32, device="cuda"), torch.tensor([28, 29], dtype=torch.int32, device="cuda")

    def step():
        st.st_norm_rows(x, layer.norm, residual, buffers=rows)
        heads = st.st_project(rows.q, rows.scale, layer.qkv.w, layer.qkv.scale, layer.qkv.adapters, tenants, buffers=qkv).view(n, 8, 64)
        st.st_rotate(heads[:, :4], heads[:, 4:6], positions, layer.freqs, layer.sections, out=(heads[:, :4], heads[:, 4:6]))
        st.st_kv_append(store.cache, batch, heads[:, 4:6], heads[:, 6:])
        out = st.st_kv_attend(store.cache, batch, heads[:, :4], buffers=attended)
        st.st_norm_rows(out.view(n, 256), normalise=False, buffers=seen)
        out = st.st_project(seen.q, seen.scale, layer.out.w, layer.out.scale, layer.out.adapters, tenants, buffers=back)
        st.st_norm_rows(out, layer.norm, rows.total, buffers=last)
        st.st_kv_copy(store.cache, store.cache, src, dst)

    results = lambda: [t.clone() for t in (last.q, last.scale, last.total, qkv.out, store.cache.k[28:], store.cache.v_scale[28:])]  # noqa: E731
    assert not (store.shares[28:] > 0).any()
    step()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            step()
    kept = [t.clone() for t in (store.cache.k, store.cache.v, store.cache.k_scale, store.cache.v_scale, store.cache.bounds)]

    def rewind():
        for t, was in zip((store.cache.k, store.cache.v, store.cache.k_scale, store.cache.v_scale, store.cache.bounds), kept):
            t.copy_(was)

    for turn in range(4):
        x.copy_(normal(n, 192) * (turn + 1))
        residual.copy_(normal(n, 192))
        positions.add_(turn)
        rewind()
        step()
        want = results()
        torch.cuda.synchronize()
        for g in graphs:
            rewind()
            g.replay()
            assert all(torch.equal(a, b) for a, b in zip(results(), want))


def test_calls_on_another_stream(monkeypatch):
    """What a call allocates on the stream it names is not handed out before the work there is done, and its results stay while the
    current stream reads them."""
    gen = torch.Generator(device="cuda").manual_seed(12)
    layer, normal = make(gen, torch.bfloat16, width=2048)
    x, residual = normal(300, 2048), normal(300, 2048)
    tenants = (torch.arange(300, device="cuda") % 3).int()
    positions = torch.stack([torch.arange(300), torch.arange(300)]).int().cuda()
    rows = st.st_norm_rows(x, layer.norm, residual, y=True)
    qkv = st.st_project(rows.q, rows.scale, layer.qkv.w, layer.qkv.scale, layer.qkv.adapters, tenants)
    heads = qkv.view(300, 8, 64)
    calls = [lambda **kw: st.st_norm_rows(x, layer.norm, residual, y=True, **kw),
             lambda **kw: st.st_project(rows.q, rows.scale, layer.qkv.w, layer.qkv.scale, layer.qkv.adapters, tenants, **kw),
             lambda **kw: st.st_rotate(heads[:, :4], heads[:, 4:6], positions, layer.freqs, layer.sections, **kw)]
    side = torch.cuda.Stream()
    for call in calls:
        want = call()
        want = [t for t in (want if isinstance(want, tuple) else (want,)) if t is not None]
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        kept = busy(side)
        asked, empty = [], torch.empty
        monkeypatch.setattr(torch, "empty", lambda *a, **kw: note(asked, empty(*a, **kw)))
        got = call(stream=side)
        monkeypatch.undo()
        got = [t for t in (got if isinstance(got, tuple) else (got,)) if t is not None]
        assert asked and not side.query()
        now = [torch.empty(size, dtype=torch.uint8, device="cuda") for size in (1 << 16, 1 << 18, 1 << 20, 1 << 22)]
        assert not {t.data_ptr() for t in now} & set(asked)
        for t in now:
            t.fill_(0xFF)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        again = busy(torch.cuda.current_stream())
        later = [t.clone() for t in got]
        sizes = [(t.shape, t.dtype) for t in got]
        del got
        with torch.cuda.stream(side):
            others = [torch.empty(shape, dtype=dtype, device="cuda").fill_(1) for shape, dtype in sizes]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(later, want))
        del kept, again, others


def test_python_calls_that_are_refused():
    """Types, shapes and strides that the library could not see."""
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    q8, scale, w, ws = x.char(), torch.ones(4, device="cuda"), torch.zeros((32, 64), dtype=torch.int8, device="cuda"), torch.ones(32, device="cuda")
    good = st.Adapters(torch.zeros((2, 8, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 32, 8), dtype=torch.bfloat16, device="cuda"),
                       torch.ones(2, device="cuda"))
    of = torch.zeros(4, dtype=torch.int32, device="cuda")
    heads = x.view(4, 1, 64)
    pos, freqs = torch.zeros((1, 4), dtype=torch.int32, device="cuda"), torch.ones(16, dtype=torch.float64, device="cuda")
    bad = [lambda: st.st_norm_rows(x.cpu()), lambda: st.st_norm_rows(x.double()), lambda: st.st_norm_rows(x[0]), lambda: st.st_norm_rows(x.t()),
           lambda: st.st_norm_rows(x, x[0].float()), lambda: st.st_norm_rows(x, x[0, :32].contiguous()), lambda: st.st_norm_rows(x, residual=x[:3]),
           lambda: st.st_norm_rows(x, total=x.float()), lambda: st.st_norm_rows(x, q=False),
           lambda: st.st_norm_rows(x, buffers=st.RowBuffers(5, 64, torch.bfloat16)), lambda: st.st_norm_rows(x, eps=0.0),
           lambda: st.st_norm_rows(x[:, :24]), lambda: st.st_norm_rows(x[:, 4:52]),
           lambda: st.st_project(q8[:, :32], scale, w[:, :32], ws), lambda: st.st_project(q8, scale[:3], w, ws), lambda: st.st_project(q8, scale, w, ws, good),
           lambda: st.st_project(q8, scale, w, ws, None, of), lambda: st.st_project(q8, scale, w, ws, good, of.long()),
           lambda: st.st_project(q8, scale, w, ws, good, of[:3]), lambda: st.st_project(q8, scale, w, ws, good, of, dtype=torch.float16),
           lambda: st.st_project(q8, scale, w[:16], ws[:16], good, of), lambda: st.st_project(q8, scale, w, ws, dtype=torch.float32),
           lambda: st.st_project(q8, scale, w, ws, out=torch.zeros((4, 48), dtype=torch.bfloat16, device="cuda")),
           lambda: st.st_project(q8, scale, w, ws, good, of, buffers=st.ProjectBuffers(1, 64, 32)),
           lambda: st.Adapters(good.a, good.b[:1], good.alpha), lambda: st.Adapters(good.a, good.b.half(), good.alpha),
           lambda: st.Adapters(good.a.float(), good.b, good.alpha), lambda: st.Adapters(good.a, good.b.transpose(1, 2), good.alpha),
           lambda: st.st_rotate(None, None, pos, freqs, (16,)), lambda: st.st_rotate(heads, heads[:3], pos, freqs, (16,)),
           lambda: st.st_rotate(heads, heads.half(), pos, freqs, (16,)), lambda: st.st_rotate(heads, None, pos, freqs, (8,)),
           lambda: st.st_rotate(heads, None, pos, freqs, (8, 8)), lambda: st.st_rotate(heads, None, pos.long(), freqs, (16,)),
           lambda: st.st_rotate(heads, None, pos, freqs.float(), (16,)), lambda: st.st_rotate(heads, None, pos, freqs, (16,), out=(None, heads)),
           lambda: st.st_rotate(heads, None, pos, freqs, (16,), out=(heads[:, :, :32], None)),
           lambda: st.st_rotate(x.view(1, 64, 4).transpose(1, 2), None, pos[:, :1].contiguous(), freqs, (16,))]
    cache = st.KvCache.empty(3, 1, 64)
    bad += [lambda: st.st_kv_copy(cache, cache, of, of[:2]), lambda: st.st_kv_copy(cache, cache, of.long(), of.long()),
            lambda: st.st_kv_copy(cache, st.KvCache.empty(3, 2, 64), of, of), lambda: st.st_kv_copy(cache, cache, of[None], of[None])]
    for i, call in enumerate(bad):
        with pytest.raises((TypeError, ValueError, st.StError)):
            call()
            print("not refused:", i)


@pytest.mark.parametrize("n_rows", [1, 40, 300, 2100, 9000])
def test_captured_projections_of_each_route_replay_as_they_run(n_rows):
    """Norm, projection and rotation of few and of many rows, ordered by adapter or not, replayed with other rows and tenants."""
    gen = torch.Generator(device="cuda").manual_seed(n_rows)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda").bfloat16()

    k, heads, d, count = 272, 9, 64, 7
    n = heads * d
    w = st.st_norm_rows(normal(n, k), normalise=False)
    adapters = st.Adapters(normal(count, 24, k), normal(count, n, 24), torch.rand(count, generator=gen, device="cuda"))
    x, weight, of = normal(n_rows, k), normal(k), torch.zeros(n_rows, dtype=torch.int32, device="cuda")
    positions, freqs = torch.zeros((1, n_rows), dtype=torch.int32, device="cuda"), torch.rand(24, dtype=torch.float64, device="cuda")
    rows, buffers = st.RowBuffers(n_rows, k, torch.bfloat16), st.ProjectBuffers(n_rows, k, n, torch.bfloat16, adapters)

    def step():
        st.st_norm_rows(x, weight, buffers=rows)
        out = st.st_project(rows.q, rows.scale, w.q, w.scale, adapters, of, buffers=buffers).view(n_rows, heads, d)
        st.st_rotate(out[:, :8], out[:, 8:], positions, freqs, (24,), interleaved=True, out=(out[:, :8], out[:, 8:]))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        x.copy_(normal(n_rows, k))
        of.copy_(torch.randint(-1, count + 1, (n_rows,), generator=gen, device="cuda"))
        positions.copy_(torch.randint(0, 1 << 30, (1, n_rows), generator=gen, device="cuda"))
        step()
        want = rows.q.clone(), rows.scale.clone(), buffers.out.clone()
        buffers.out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip((rows.q, rows.scale, buffers.out), want))


def test_layer_of_no_users_and_of_users_without_tokens():
    gen = torch.Generator(device="cuda").manual_seed(4)
    layer, normal = make(gen, torch.bfloat16)
    store = HistoryStore(3, 10, 2, 64, 3)
    none = torch.zeros((2, 0), dtype=torch.int32, device="cuda")
    tenants = torch.zeros(0, dtype=torch.int32, device="cuda")
    for append in (True, False):
        out, total = layer(store, [], normal(0, 192), none, [], tenants, normal(0, 192), append=append)
        assert out.shape == total.shape == (0, 192)
    layer.take_in(store, [], normal(0, 192), none, [], tenants)
    # a user without an event, and candidates of one that has no history
    positions = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    out, _ = layer(store, [0, 1], normal(3, 192), positions, [3, 0], torch.zeros(3, dtype=torch.int32, device="cuda"))
    assert store.lengths.tolist() == [3, 0, 0] and torch.isfinite(out.float()).all()
    out, _ = layer(store, [2], normal(3, 192), positions, [3], torch.zeros(3, dtype=torch.int32, device="cuda"), append=False)
    assert (out == 0).all()
