"""The operators of a layer around the cached histories through the C ABI against the plain implementation in 64 bits
(layer_reference, which derives the bounds).  Sums with the residual, integers and copied pages are compared bit for bit."""
import numpy as np
import pytest
import torch

from paper_2511_14881_amd import binding as st
from tests import layer_reference as R

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)


def rows_of(rng, n, d, dtype, size=1.0):
    x = rng.normal(0, 1, (n, d)) * np.exp(rng.normal(0, 1, (n, 1))) * size
    return torch.from_numpy(x.astype(np.float32)).to(R.TYPES[dtype])


def spread(t, stride, offset=0):
    """The tensor's rows, `stride` elements apart, in memory filled with something else."""
    n, width = t.shape[0], t[0].numel()
    base = torch.full((offset + max(n, 1) * stride,), 77.0, dtype=t.dtype, device="cuda")
    shape, strides = (n, *t.shape[1:]), (stride, *t[0].contiguous().stride())
    view = base.as_strided(shape, strides, offset)
    view.copy_(t)
    return view


NORMS = [
    # dtype, rows, d, weight, residual, y, normalise
    ("bf16", 1, 16, True, True, True, True),
    ("f16", 5, 64, True, False, False, True),
    ("f32", 17, 128, False, True, True, True),
    ("bf16", 33, 144, True, True, False, True),
    ("f32", 3, 512, True, True, True, True),
    ("f16", 9, 528, True, True, True, True),
    ("bf16", 70, 1008, True, True, True, True),
    ("f16", 4, 1040, False, False, True, True),
    ("bf16", 5, 2048, True, True, False, False),
    ("f16", 3, 2064, True, True, True, True),
    ("f32", 2, 4112, True, True, True, True),
    ("bf16", 3, 8192, True, False, True, True),
    ("f16", 2, 8208, True, True, True, True),
    ("f32", 2, 16384, True, True, True, True),
    ("bf16", 1, 16384, True, True, True, True),
]


@pytest.mark.parametrize("case", range(len(NORMS)))
def test_norm_matches_plain(case):
    dtype, n, d, has_weight, has_residual, y, normalise = NORMS[case]
    say(f"[layer] norm case {case}: {NORMS[case]}")
    rng = np.random.default_rng(case)
    x, residual = rows_of(rng, n, d, dtype), rows_of(rng, n, d, dtype, 0.5) if has_residual else None
    if n > 2:
        x[1] = 0
        if has_residual:
            residual[1] = 0
    weight = rows_of(rng, 1, d, dtype)[0].contiguous() if has_weight else None
    h, q, unit, rms, t = R.norm(x, weight, residual, 1e-5, normalise)
    xs = spread(x, d + 8 * (case % 3))
    rs = spread(residual, d + 8 * (case % 2), 16) if has_residual else None
    got = st.st_norm_rows(xs, None if weight is None else weight.cuda(), rs, eps=1e-5, normalise=normalise, y=y)
    torch.cuda.synchronize()
    if has_residual:
        assert torch.equal(got.total.cpu(), h)
    else:
        assert got.total is None
    assert np.array_equal(got.q.cpu().numpy(), q)
    off = R.norm_bound(d) if normalise else R.F32
    assert np.all(np.abs(got.scale.cpu().numpy() - unit * rms) <= off * unit * rms + 2.0 ** -149)
    assert torch.equal(xs.cpu(), x)
    if y:
        want = t * rms[:, None]
        half = R.half_step(dtype)
        assert np.all(np.abs(got.y.double().cpu().numpy() - want) <= np.abs(want) * (half + 2 * off) + R.least(dtype))
    else:
        assert got.y is None


def test_norm_in_place_and_single_outputs():
    rng = np.random.default_rng(50)
    x, r = rows_of(rng, 37, 320, "bf16"), rows_of(rng, 37, 320, "bf16")
    weight = rows_of(rng, 1, 320, "bf16")[0].cuda()
    want = st.st_norm_rows(x.cuda(), weight, r.cuda(), y=True)
    for place in ("x", "residual"):
        a, b = spread(x, 336), spread(r, 328)
        got = st.st_norm_rows(a, weight, b, total=a if place == "x" else b)
        assert torch.equal(got.total, want.total) and got.total is (a if place == "x" else b)
        assert torch.equal(got.q, want.q) and torch.equal(got.scale, want.scale)
    only = st.st_norm_rows(x.cuda(), weight, r.cuda(), q=False, y=True)
    assert only.q is None and only.scale is None and torch.equal(only.y, want.y) and torch.equal(only.total, want.total)
    buffers = st.RowBuffers(37, 320, torch.bfloat16, y=True)
    got = st.st_norm_rows(x.cuda(), weight, r.cuda(), buffers=buffers)
    assert got.total is None and got.q is buffers.q and torch.equal(got.y, want.y)
    none = st.st_norm_rows(x[:0].cuda(), weight)
    assert none.q.shape == (0, 320)


def test_norm_of_extreme_rows():
    """Rows whose squares leave fp32 (on both sides), and rows that hold what is no number."""
    d = 272
    rng = np.random.default_rng(51)
    for dtype in ("bf16", "f32"):
        x = rows_of(rng, 6, d, dtype)
        x = x / x.float().abs().amax(1, keepdim=True).to(x.dtype)
        x[1] = (x[1].double() * 2.0 ** 127).to(x.dtype)
        x[2] = (x[2].double() * 2.0 ** -90).to(x.dtype)
        x[3, 5], x[4, 100], x[5, 7] = float("nan"), float("inf"), float("-inf")
        weight = rows_of(rng, 1, d, dtype)[0]
        got = st.st_norm_rows(x.cuda(), weight.cuda(), eps=1e-6, y=True)
        fine = x[:3].clone()
        fine[1] = (fine[1].double() * 2.0 ** -70).to(x.dtype)
        _, q, unit, rms, t = R.norm(fine, weight, None, 1e-6, True)
        assert np.array_equal(got.q[:3].cpu().numpy(), q)
        assert (got.q[3:] == 0).all() and torch.isnan(got.scale[3:]).all() and torch.isnan(got.y[3:].float()).all()
        off = R.norm_bound(d)
        assert np.all(np.abs(got.scale[:3].cpu().numpy() - unit * rms) <= off * unit * rms + 2.0 ** -149)
        want = t * rms[:, None]
        assert np.all(np.abs(got.y[:3].double().cpu().numpy() - want) <= np.abs(want) * (R.half_step(dtype) + 2 * off) + R.least(dtype))
    # a sum that leaves fp16
    big = torch.full((1, 32), 40000.0, dtype=torch.float16, device="cuda")
    got = st.st_norm_rows(big, residual=big)
    assert torch.isinf(got.total).all() and torch.isnan(got.scale).all() and (got.q == 0).all()


def integers(rng, *shape):
    return torch.from_numpy(rng.integers(-128, 128, shape).astype(np.int8))


def some_adapters(rng, count, rank, k, n, dtype):
    a = torch.from_numpy(rng.normal(0, k ** -0.5, (count, rank, k)).astype(np.float32)).to(R.TYPES[dtype])
    b = torch.from_numpy(rng.normal(0, 0.3, (count, n, rank)).astype(np.float32)).to(R.TYPES[dtype])
    return a, b, torch.from_numpy(rng.uniform(0.2, 2.0, count).astype(np.float32))


PROJECTIONS = [
    # dtype, rows, k, n, adapters, rank, order
    ("bf16", 1, 16, 16, 0, 0, None),
    ("f16", 1, 64, 48, 3, 8, "mixed"),
    ("bf16", 3, 512, 1024, 8, 16, "mixed"),
    ("f16", 16, 80, 144, 1, 16, "runs"),
    ("bf16", 17, 128, 128, 5, 24, "mixed"),
    ("f16", 33, 1040, 272, 40, 32, "mixed"),
    ("bf16", 64, 2048, 160, 64, 16, "mixed"),
    ("f16", 65, 208, 336, 2, 128, "runs"),
    ("bf16", 127, 96, 1296, 0, 0, None),
    ("f16", 130, 656, 1040, 7, 40, "mixed"),
    ("bf16", 200, 4096, 256, 3, 64, "runs"),
    ("bf16", 257, 1040, 528, 16, 72, "mixed"),
    ("f16", 300, 16384, 32, 2, 8, "none"),
    ("bf16", 515, 320, 784, 100, 16, "runs"),
    ("f16", 1025, 144, 272, 11, 104, "mixed"),
    ("bf16", 2049, 128, 512, 4, 120, "runs"),
    ("bf16", 600, 64, 64, 5000, 8, "mixed"),  # more adapters than the order has buckets
    ("f16", 2, 1008, 80, 2, 16, "mixed"),
    # k that ends in each of the chunks a part's loads run ahead by
    ("bf16", 40, 4624, 32, 3, 16, "mixed"),
    ("f16", 70, 5152, 32, 3, 64, "mixed"),
    ("bf16", 2100, 4720, 32, 2, 32, "runs"),
    ("f16", 2100, 2592, 32, 6, 128, "mixed"),
    ("bf16", 1, 992, 48, 4, 32, "mixed"),
    # several workgroups of 64 rows, and rows or columns beyond what those take
    ("bf16", 100, 512, 4096, 9, 24, "mixed"),
    ("f16", 384, 272, 1344, 5, 64, "mixed"),
    ("f16", 384, 272, 1360, 5, 64, "mixed"),
    ("bf16", 190, 272, 144, 3, 128, "mixed"),
    ("bf16", 200, 272, 144, 3, 128, "mixed"),
    ("f16", 65, 64, 8224, 6, 16, "mixed"),
    ("f16", 395, 208, 336, 2, 128, "runs"),
    ("bf16", 391, 96, 1296, 0, 0, None),
    ("f16", 410, 656, 1040, 4, 40, "mixed"),
    ("bf16", 400, 4096, 256, 3, 64, "runs"),
    ("bf16", 449, 1040, 528, 16, 72, "mixed"),
    ("f16", 390, 16384, 32, 2, 8, "none"),
    ("f16", 386, 5152, 32, 3, 64, "mixed"),
]


def project_case(cases, case):
    dtype, rows, k, n, count, rank, order = cases[case]
    rng = np.random.default_rng(1000 + case)
    x, w = integers(rng, rows, k), integers(rng, n, k)
    xs = torch.from_numpy(np.exp(rng.normal(-4, 1, rows)).astype(np.float32))
    ws = torch.from_numpy(np.exp(rng.normal(-6, 1, n)).astype(np.float32))
    args = (x, xs, w, ws)
    if count:
        of = rng.integers(-2, count + 2, rows) if order == "mixed" else np.arange(rows) * count // rows if order == "runs" else np.full(rows, count)
        args += (*some_adapters(rng, count, rank, k, n, dtype), torch.from_numpy(of.astype(np.int32)))
    return dtype, args


def call(args, **kw):
    x, xs, w, ws, *rest = (t.cuda() for t in args)
    return st.st_project(x, xs, w, ws, st.Adapters(*rest[:3]) if rest else None, rest[3] if rest else None, **kw)


@pytest.mark.parametrize("case", range(len(PROJECTIONS)))
def test_projection_matches_plain(case):
    say(f"[layer] projection case {case}: {PROJECTIONS[case]}")
    dtype, args = project_case(PROJECTIONS, case)
    n_rows, n = args[0].shape[0], args[2].shape[0]
    out = torch.full((n_rows + 1, n + 8 * (case % 3)), 7.0, dtype=R.TYPES[dtype], device="cuda")
    got = call(args, out=out[:n_rows, :n])
    torch.cuda.synchronize()
    want, bound = R.project(*args, dtype=dtype)
    off = np.abs(got.double().cpu().numpy() - want)
    assert np.isfinite(off).all()
    over = off - bound
    assert over.max() <= 0, f"off by {off.max()} at {np.unravel_index(over.argmax(), over.shape)}"
    assert (out[n_rows] == 7.0).all() and (out[:, n:] == 7.0).all()  # what lies behind a row and behind the rows
    assert torch.equal(call(args, dtype=R.TYPES[dtype]), got)  # the same bits again


LARGE = [
    # dtype, rows, k, n, adapters, rank, order: tiles of each edge, with rows and columns behind the last whole tile
    ("f16", 1030, 144, 8208, 6, 16, "mixed"),
    ("bf16", 2100, 528, 5136, 3, 24, "mixed"),
    ("bf16", 3000, 208, 4112, 16, 128, "runs"),
    ("f16", 2060, 4112, 5136, 9, 8, "mixed"),
    ("bf16", 4100, 1040, 5152, 300, 24, "mixed"),
    ("f16", 16400, 256, 1040, 0, 0, None),
    ("bf16", 2500, 64, 1040, 4, 16, "runs"),
    ("bf16", 2300, 2064, 288, 2, 72, "mixed"),
    ("f16", 2050, 128, 16, 3, 16, "none"),
]


@pytest.mark.parametrize("case", range(len(LARGE)))
def test_large_projection_matches_plain(case):
    """Some rows of calls that take the larger tiles."""
    say(f"[layer] large projection case {case}: {LARGE[case]}, {st.st_project_host_plan(*LARGE[case][1:6])}")
    dtype, args = project_case(LARGE, case)
    n_rows, n = args[0].shape[0], args[2].shape[0]
    out = torch.full((n_rows + 1, n + 8), 7.0, dtype=R.TYPES[dtype], device="cuda")
    got = call(args, out=out[:n_rows, :n])
    torch.cuda.synchronize()
    rng = np.random.default_rng(case)
    some = np.unique(np.concatenate([rng.integers(0, n_rows, 60), [0, 31, 32, n_rows - 1, n_rows - 2]]))
    want, bound = R.project(*(t[some] if i in (0, 1, 7) else t for i, t in enumerate(args)), dtype=dtype)
    off = np.abs(got[torch.from_numpy(some).cuda()].double().cpu().numpy() - want)
    over = off - bound
    assert over.max() <= 0, f"off by {off.max()} at {np.unravel_index(over.argmax(), over.shape)}"
    assert (out[n_rows] == 7.0).all() and (out[:, n:] == 7.0).all() and torch.isfinite(got.float()).all()
    # the rest by calls of fewer rows, which run otherwise: the same bits
    for first in range(0, n_rows, 1000):
        last = min(first + 60, n_rows)
        part = call(tuple(t[first:last] if i in (0, 1, 7) else t for i, t in enumerate(args)), dtype=R.TYPES[dtype])
        assert torch.equal(part, got[first:last])


@pytest.mark.parametrize("case", [2, 5, 9, 11, 14, 24, 25, 27, 33])
def test_projection_of_a_row_does_not_depend_on_others(case):
    dtype, args = project_case(PROJECTIONS, case)
    want = call(args, dtype=R.TYPES[dtype])
    order = torch.from_numpy(np.random.default_rng(7).permutation(args[0].shape[0]))
    got = call((args[0][order], args[1][order], *args[2:7], args[7][order]), dtype=R.TYPES[dtype])
    assert torch.equal(got, want[order.cuda()])
    some = order[:5]
    got = call((args[0][some], args[1][some], *args[2:7], args[7][some]), dtype=R.TYPES[dtype])
    assert torch.equal(got, want[some.cuda()])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_projection_of_rows_of_any_size(dtype):
    """Scales from 2^-60 to 2^60, in fp16 too, where inner values of their own size would not fit; zeros; a scale that is no number."""
    rng = np.random.default_rng(77)
    rows, k, n = 20, 192, 64
    x, w = integers(rng, rows, k), integers(rng, n, k)
    x[4] = 0
    xs = torch.from_numpy(np.ldexp(1.0, rng.integers(-60, 60, rows)).astype(np.float32))
    if dtype == "f16":  # whose outputs end at 65504
        xs.clamp_(max=2.0 ** -8)
    xs[7] = float("nan")
    ws = torch.full((n,), 2.0 ** -14)
    a, b, alpha = some_adapters(rng, 3, 16, k, n, dtype)
    b *= 2.0 ** -8
    of = torch.from_numpy((np.arange(rows) % 3).astype(np.int32))
    args = (x, xs, w, ws, a, b, alpha, of)
    got = call(args).double().cpu().numpy()
    want, bound = R.project(*args, dtype=dtype)
    fine = np.arange(rows) != 7
    assert np.isnan(got[7]).all() and np.all(np.abs(got - want)[fine] <= bound[fine])


ROTATIONS = [
    # dtype, tokens, q heads, k heads, d, sections, interleaved, inverse
    ("bf16", 1, 4, 1, 64, (16, 16), False, False),
    ("f16", 7, 1, 1, 96, (48,), True, False),
    ("bf16", 130, 8, 2, 128, (30, 17, 17), False, False),
    ("f16", 65, 5, 1, 128, (40, 8), True, False),
    ("bf16", 33, 3, 3, 256, (8,), False, True),
    ("f16", 50, 16, 4, 64, (5, 0, 11, 8), False, True),
    ("bf16", 9, 2, 1, 16, (8,), True, False),
    ("bf16", 3, 40, 8, 512, (100, 100, 56), False, False),
    ("f16", 12, 1, 0, 24, (8,), False, False),
    ("bf16", 12, 0, 3, 128, (20, 20, 24), True, True),
]


@pytest.mark.parametrize("case", range(len(ROTATIONS)))
def test_rotation_matches_plain(case):
    dtype, n, qh, kh, d, sections, interleaved, inverse = ROTATIONS[case]
    say(f"[layer] rotation case {case}: {ROTATIONS[case]}")
    rng = np.random.default_rng(2000 + case)
    pairs = sum(sections)
    positions = np.stack([rng.integers(0, 5000, n), rng.integers(1_600_000_000, 2 ** 31 - 1, n), rng.integers(-2 ** 31, 0, n),
                          rng.integers(0, 2, n)][:len(sections)]).astype(np.int32)
    freqs = torch.from_numpy(np.exp(rng.uniform(np.log(1e-9), 0.0, pairs)))
    pos = torch.from_numpy(positions)
    qkv = torch.from_numpy(rng.normal(0, 2, (n, qh + 2 * kh, d)).astype(np.float32)).to(R.TYPES[dtype])
    held = spread(qkv, (qh + 2 * kh) * d + 8 * (case % 2))
    q, k = (held[:, :qh] if qh else None), (held[:, qh:qh + kh] if kh else None)
    args = (pos.cuda(), freqs.cuda(), sections, interleaved, inverse)
    got = st.st_rotate(q, k, *args)
    torch.cuda.synchronize()
    for rows, out in ((q, got[0]), (k, got[1])):
        if rows is None:
            assert out is None
            continue
        want, bound = R.rotate(rows.cpu(), pos, freqs, sections, interleaved, inverse, dtype)
        off = np.abs(out.double().cpu().numpy() - want) - bound
        assert off.max() <= 0, f"{off.max()} over the bound at {np.unravel_index(off.argmax(), off.shape)}"
    assert torch.equal(held.cpu(), qkv)
    # in place: the same bits, and the values beside them stay
    again = st.st_rotate(q, k, *args, out=(q, k))
    for a, b in zip(again, got):
        assert b is None or torch.equal(a, b)
    assert torch.equal(held[:, qh + kh:].cpu(), qkv[:, qh + kh:])


def test_rotation_and_back():
    """The inverse takes a rotated row back, and is the transpose of the rotation: a gradient against differences in 64 bits."""
    rng = np.random.default_rng(9)
    n, d, sections = 40, 64, (20, 12)
    pos = torch.from_numpy(rng.integers(0, 2 ** 31 - 1, (2, n)).astype(np.int32))
    freqs = torch.from_numpy(np.exp(rng.uniform(-9, 0, 32)))
    x, g = (torch.from_numpy(rng.normal(0, 1, (n, 2, d)).astype(np.float32)).half() for _ in range(2))
    args = (pos.cuda(), freqs.cuda(), sections)
    there = st.st_rotate(x.cuda(), None, *args)[0]
    back = st.st_rotate(there, None, *args, inverse=True)[0]
    # two roundings of values up to |x| + |y|, and cos, sin off by 2^-20 twice
    pair = np.abs(x.double().numpy())
    size = pair + np.roll(pair, 32, -1)
    assert np.all(np.abs(back.double().cpu().numpy() - x.double().numpy()) <= size * (2 * 2.0 ** -11 * 1.01 + 2 * 2.0 ** -20) + 2.0 ** -23)
    grad = st.st_rotate(g.cuda(), None, *args, inverse=True)[0].double().cpu().numpy()
    step = 2.0 ** -12
    for t, h, c in ((0, 0, 0), (3, 1, 31), (17, 0, 32), (39, 1, 63), (20, 0, 45)):
        sides = []
        for s in (step, -step):
            moved = x.double().clone()
            moved[t, h, c] += s
            sides.append((R.rotate(moved, pos, freqs, sections, False, False, "f16")[0] * g.double().numpy()).sum())
        slope = (sides[0] - sides[1]) / (2 * step)
        other = np.abs(g.double().numpy()[t, h, c]) + np.abs(g.double().numpy()[t, h, (c + 32) % 64])
        # the slope's sums cancel: some 5000 values rounded to 2^-53, over two steps
        assert abs(grad[t, h, c] - slope) <= other * (2.0 ** -11 + 2.0 ** -19) + 2.0 ** -24 + 5120 * 8 * 2.0 ** -53 / step


def pages(rng, n, heads, d):
    return st.KvCache(integers(rng, n, heads, 64, d).cuda(), integers(rng, n, heads, d, 64).cuda(),
                      torch.from_numpy(rng.uniform(0, 1, (n, heads)).astype(np.float32)).cuda(),
                      torch.from_numpy(rng.uniform(0, 1, (n, heads)).astype(np.float32)).cuda(), integers(rng, n, heads, 2, d).cuda())


def parts(cache):
    return [t.cpu().clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.bounds)]


@pytest.mark.parametrize("heads,d", [(1, 64), (3, 96), (8, 128), (2, 256), (300, 64)])
def test_copied_pages(heads, d):
    say(f"[layer] copy {heads} x {d}")
    rng = np.random.default_rng(heads * 1000 + d)
    one, other = pages(rng, 11, heads, d), pages(rng, 7, heads, d)
    src = [4, 0, 9, -1, 3, 11, 2, 5, 2 ** 31 - 1]
    dst = [1, 6, 8, 2, -7, 10, 7, 12, 0]
    # one cache: page 10 is no source's, 11 and beyond are no pages
    want = parts(one)
    for a, b in zip(src, dst):
        if 0 <= a < 11 and 0 <= b < 11:
            for t in want:
                t[b] = t[a]
    lists = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (src, dst)]
    st.st_kv_copy(one, one, *lists)
    assert all(torch.equal(a, b) for a, b in zip(parts(one), want))
    # two caches of different sizes
    want = parts(other)
    for a, b in zip(src, dst):
        if 0 <= a < 11 and 0 <= b < 7:
            for t, s in zip(want, parts(one)):
                t[b] = s[a]
    st.st_kv_copy(one, other, *lists)
    assert all(torch.equal(a, b) for a, b in zip(parts(other), want))
    st.st_kv_copy(one, one, lists[0][:0], lists[1][:0])


@pytest.mark.parametrize("case", [("bf16", 17, 128, 128, 5, 24), ("f16", 64, 512, 80, 20, 16), ("bf16", 2, 512, 64, 2, 16), ("f16", 130, 208, 144, 4, 40), ("f16", 420, 208, 144, 4, 40),
                                  ("bf16", 600, 96, 272, 9, 16), ("f16", 2100, 128, 5136, 3, 24), ("bf16", 4100, 64, 5152, 30, 8)])
def test_projection_beside_adapters_that_are_no_numbers(case):
    """Infinities and NaN in one tenant's adapter, another's factor that is none: the other tenants' rows keep their bits."""
    say(f"[layer] projection beside bad adapters {case}")
    dtype, rows, k, n, count, rank = case
    args = project_case([(*case, "mixed")], 0)[1]
    args[7][:count] = torch.arange(count, dtype=torch.int32)[: rows]
    want = call(args, dtype=R.TYPES[dtype])
    a, b, alpha = (t.clone() for t in args[4:7])
    b[0, 0::3], b[0, 1::3] = float("inf"), float("nan")
    a[0, 0], a[0, -1] = float("-inf"), float("nan")
    alpha[count - 1] = float("nan")
    got = call((*args[:4], a, b, alpha, args[7]), dtype=R.TYPES[dtype])
    kept = ((args[7] != 0) & (args[7] != count - 1)).cuda()
    assert torch.equal(got[kept], want[kept]) and not torch.isfinite(got[~kept][:, 0]).any()


def test_offsets_beyond_32_bits():
    """Rows, heads, adapters, outputs and pages that lie more than 2^31 elements behind the first: as in a call of their own."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    n, d, last = 131072 + 40, 16384, 70
    say("[layer] norm beyond 2^31 values")
    x = torch.empty((n, d), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    rows, own = st.st_norm_rows(x), st.st_norm_rows(x[-last:].clone())
    assert torch.equal(rows.q[-last:], own.q) and torch.equal(rows.scale[-last:], own.scale)
    del x
    say("[layer] projection of more than 2^31 values")
    w, ws = torch.randint(-128, 128, (32, d), dtype=torch.int8, device="cuda"), torch.full((32,), 2.0 ** -12, device="cuda")
    ad = st.Adapters(torch.randn((6, 8, d), device="cuda").bfloat16(), torch.randn((6, 32, 8), device="cuda").bfloat16(), torch.ones(6, device="cuda"))
    of = torch.arange(n, dtype=torch.int32, device="cuda") % 7
    got = st.st_project(rows.q, rows.scale, w, ws, ad, of)
    assert torch.equal(got[-last:], st.st_project(own.q, own.scale, w, ws, ad, of[-last:].clone()))
    del rows, got
    say("[layer] adapters beyond 2^31 values")
    count, k = st.ST_MAX_ADAPTERS, 4112
    a, b = (torch.empty(shape, dtype=torch.float16, device="cuda").normal_(generator=gen) for shape in ((count, 8, k), (count, k, 8)))
    alpha = torch.rand(count, device="cuda", generator=gen)
    w, ws = torch.randint(-128, 128, (k, k), dtype=torch.int8, device="cuda"), torch.full((k,), 2.0 ** -16, device="cuda")
    many = st.Adapters(a, b, alpha)
    few = st.Adapters(a[-16:].clone(), b[-16:].clone(), alpha[-16:].clone())
    for m in (1, 20, 70):
        of = torch.randint(count - 16, count, (m,), dtype=torch.int32, device="cuda")
        q, scale = torch.randint(-128, 128, (m, k), dtype=torch.int8, device="cuda"), torch.full((m,), 2.0 ** -6, device="cuda")
        assert torch.equal(st.st_project(q, scale, w, ws, many, of), st.st_project(q, scale, w, ws, few, of - (count - 16)))
    del a, b, many
    say("[layer] outputs beyond 2^31 values")
    m, stride = 16500, 131072
    base = torch.zeros((m * stride,), dtype=torch.bfloat16, device="cuda")
    q, scale = torch.randint(-128, 128, (m, 64), dtype=torch.int8, device="cuda"), torch.full((m,), 2.0 ** -6, device="cuda")
    w, ws = w[:64, :64].contiguous(), ws[:64].contiguous()
    got = st.st_project(q, scale, w, ws, out=base.as_strided((m, 64), (stride, 1)))
    assert torch.equal(got, st.st_project(q, scale, w, ws))
    del base, got
    say("[layer] rotation beyond 2^31 values")
    n, heads, d = 262144 + 40, 64, 128
    q = torch.empty((n, heads, d), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    pos = torch.randint(0, 1 << 30, (1, n), dtype=torch.int32, device="cuda")
    freqs = torch.rand(32, dtype=torch.float64, device="cuda")
    want = st.st_rotate(q[-last:].clone(), None, pos[:, -last:].contiguous(), freqs, (32,))[0]
    st.st_rotate(q, None, pos, freqs, (32,), out=(q, None))
    assert torch.equal(q[-last:], want)
    del q
    say("[layer] pages beyond 2^31 bytes")
    cache = st.KvCache.empty(33000, 8, 128)
    for t in (cache.k, cache.v, cache.bounds):
        t[32990:] = torch.randint(-128, 128, t[32990:].shape, dtype=torch.int8, device="cuda")
    st.st_kv_copy(cache, cache, *(torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([32999, 32991], [1, 32980])))
    for t in (cache.k, cache.v, cache.bounds):
        assert torch.equal(t[1], t[32999]) and torch.equal(t[32980], t[32991]) and t[1].any()
