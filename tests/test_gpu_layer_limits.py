"""The operators of a layer around the cached histories where their numbers end: inner values that cancel, adapters of any size beside their
row's own, rows at the end of a type, values behind the last of k, positions far from the first.
Bounds: layer_reference, or derived here."""
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2511_14881_amd import binding as st
from tests import layer_reference as R
from tests.test_gpu_layer import call, integers, rows_of, say

pytestmark = pytest.mark.gpu

# rows that take each route at k = 64 to 272 and few columns: one launch, few rows, several workgroups of them, tiles with and without an order
ROUTES = [2, 20, 100, 600, 2100]


# ---------------------------------------------------------------- inner values that cancel
# the exponents of an adapter's factor and of b: outputs in fp16's range, with inner values of any size (bf16's own least among them)
@pytest.mark.parametrize("dtype,size,up", [("bf16", -10, 0), ("f16", -10, 0), ("bf16", -121, 110), ("bf16", 90, -90), ("f16", 2, -12)])
@pytest.mark.parametrize("n_rows", ROUTES)
def test_projection_of_inner_values_that_cancel(n_rows, dtype, size, up):
    """Ranks in pairs of nearly the same inner value, with opposite signs behind them: what is left of a pair is some 2^-8 of either.  All sums
    before the rounding to two 16-bit halves are of integers below 2^24, with factors that are powers of two, and so exact; the halves leave
    half a step of half a step (and fp16's smallest numbers, whose half step is 2^-25 beside a row's largest value in [1, 2))."""
    say(f"[layer] cancelling inner values, {n_rows} rows, {dtype}, 2^{size}, 2^{up}")
    rng = np.random.default_rng(n_rows)
    k, n, rank, count = 64, 48, 8 if n_rows == 2 else 24, 6
    x = integers(rng, n_rows, k)
    a = rng.integers(-64, 65, (count, rank, k))
    a[:, 1::2] = np.clip(a[:, 0::2] + rng.integers(-1, 2, (count, rank // 2, k)) * (rng.random((count, rank // 2, k)) < 0.1), -64, 64)
    b = rng.integers(-64, 65, (count, n, rank))
    b[:, :, 1::2] = -b[:, :, 0::2]
    of = rng.integers(-1, count, n_rows)
    half = R.half_step(dtype)
    b = b * 2.0 ** up
    args = (x, torch.full((n_rows,), 2.0 ** -6), torch.zeros((n, k), dtype=torch.int8), torch.ones(n), torch.from_numpy(a).to(R.TYPES[dtype]),
            torch.from_numpy(b).to(R.TYPES[dtype]), torch.full((count,), 2.0 ** size), torch.from_numpy(of.astype(np.int32)))
    got = call(args).double().cpu().numpy()
    x64 = x.double().numpy()
    for i in range(count):
        rows = of == i
        inner = x64[rows] @ a[i].T.astype(np.float64) * 2.0 ** (size - 6)
        want = inner @ b[i].T
        left = half * half * np.abs(inner) + (2.0 ** -25 if dtype == "f16" else 0.0) * np.abs(inner).max(1, keepdims=True)
        off = left @ np.abs(b[i]).T + (2 * rank + 8) * R.F32 * (np.abs(inner) @ np.abs(b[i]).T)
        over = np.abs(got[rows] - want) - off - half * (np.abs(want) + off) - R.least(dtype)
        assert not rows.any() or over.max() <= 0, f"{over.max()} over the bound"
    assert (got[of < 0] == 0).all()


# ---------------------------------------------------------------- adapters of any size beside their row's own
FAR = {  # exponents: of the smallest and largest scale of a row, of the weights' scales, of the adapters' factors
    "bf16": [(6, 20, -14, (-106, -120, -149, -60, 0, 60)), (0, 20, 40, (-106, -120, -149, -60, 0, 60)), (-30, 0, -14, (-106, -120, -149, -60, 0, 60))],
    "f16": [(6, 20, -35, (-106, -120, -149, -60, -40, -31)), (60, 80, -95, (-106, -120, -149, -100, -95, -91)), (-30, 0, -16, (-106, -120, -149, -60, -30, -9))],
}


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n_rows", ROUTES)
def test_projection_with_adapters_far_below_and_above(n_rows, dtype):
    """Inner values from 2^-130 to 2^100 beside sums of products from 2^-30 to 2^80: neither term leaves fp32 for the other's sake."""
    say(f"[layer] adapters far below and above, {n_rows} rows, {dtype}")
    rng = np.random.default_rng(100 + n_rows)
    k, n, rank, count = 256, 64, 8, 6
    x, w = torch.full((n_rows, k), 127, dtype=torch.int8), integers(rng, n, k)
    w[0] = 127
    a = torch.from_numpy(rng.uniform(0.5, 1.0, (count, rank, k)).astype(np.float32)).to(R.TYPES[dtype])
    b = torch.from_numpy(rng.normal(0, 1, (count, n, rank)).astype(np.float32)).to(R.TYPES[dtype])
    of = torch.from_numpy(rng.integers(-1, count, n_rows).astype(np.int32))
    for low, high, weight, factors in FAR[dtype]:
        alpha = torch.from_numpy(np.ldexp(1.0, factors).astype(np.float32))
        xs = torch.from_numpy(np.ldexp(1.0, rng.integers(low, high + 1, n_rows)).astype(np.float32))
        args = (x, xs, w, torch.full((n,), 2.0 ** weight), a, b, alpha, of)
        got = call(args).double().cpu().numpy()
        want, bound = R.project(*args, dtype=dtype)
        assert np.isfinite(got).all()
        over = np.abs(got - want) - bound
        assert over.max() <= 0, f"{over.max()} over the bound, scales 2^{low} to 2^{high}"


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n_rows", ROUTES)
def test_projection_beside_an_adapter_that_adds_nothing(n_rows, dtype):
    """b = 0, as before the first step of its training: the outputs are those without the adapter, however large its inner values are."""
    say(f"[layer] adapters that add nothing, {n_rows} rows, {dtype}")
    rng = np.random.default_rng(200 + n_rows)
    k, n, rank, count = 128, 48, 8, 6
    x, w = integers(rng, n_rows, k), integers(rng, n, k)
    xs, ws = torch.full((n_rows,), 2.0 ** -8), torch.full((n,), 2.0 ** -8)
    a = torch.from_numpy(rng.integers(32, 65, (count, rank, k)).astype(np.float32)).to(R.TYPES[dtype])
    alpha = torch.from_numpy(np.ldexp(1.0, [-149, -100, 0, 90, 110, 113]).astype(np.float32))
    of = torch.from_numpy((np.arange(n_rows) % count).astype(np.int32))
    want = call((x, xs, w, ws), dtype=R.TYPES[dtype])
    got = call((x, xs, w, ws, a, torch.zeros((count, n, rank), dtype=R.TYPES[dtype]), alpha, of))
    assert torch.equal(got, want)


# ---------------------------------------------------------------- workspaces of more rows
def test_buffers_of_more_rows_serve_fewer():
    """192 rows of rank 128 need more than 500 or 2000 do by their own route."""
    rng = np.random.default_rng(300)
    k, n, rank, count, rows = 272, 144, 128, 4, 2000
    args = (integers(rng, rows, k), torch.full((rows,), 2.0 ** -6), integers(rng, n, k), torch.full((n,), 2.0 ** -6),
            torch.from_numpy(rng.normal(0, 1, (count, rank, k)).astype(np.float32)).bfloat16(),
            torch.from_numpy(rng.normal(0, 1, (count, n, rank)).astype(np.float32)).bfloat16(), torch.ones(count),
            torch.from_numpy((np.arange(rows) % count).astype(np.int32)))
    x, xs, w, ws, a, b, alpha, of = (t.cuda() for t in args)
    adapters = st.Adapters(a, b, alpha)
    buffers = st.ProjectBuffers(rows, k, n, torch.bfloat16, adapters)
    for m in (1, 64, 192, 193, 500, 2000):
        some = x[:m], xs[:m], w, ws, adapters, of[:m]
        assert torch.equal(st.st_project(*some, out=buffers.out[:m], buffers=buffers), st.st_project(*some))


# ---------------------------------------------------------------- rows at the end of a type
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [2048, 4208, 8192, 16384])
def test_norm_of_rows_of_the_largest_numbers(d, dtype):
    """All values near the type's largest, rows in which squares alone leave fp32, and rows on both sides of where they do."""
    say(f"[layer] norm of the largest numbers, {d}, {dtype}")
    rng = np.random.default_rng(d)
    top = float(torch.finfo(R.TYPES[dtype]).max)
    sign = torch.from_numpy(rng.choice([-1.0, 1.0], (6, d)))
    x = sign * top
    x[1] = sign[1] * 2.0 ** 100
    x[2, 1:] = 0.0
    x[3] = sign[3] * 2.0 ** 63
    x[4] = sign[4] * 2.0 ** 52
    x[5] = torch.from_numpy(rng.uniform(-top, top, d))
    x = x.to(R.TYPES[dtype])
    weight = rows_of(rng, 1, d, dtype)[0].contiguous()
    for w in (None, weight):
        got = st.st_norm_rows(x.cuda(), None if w is None else w.cuda(), y=True)
        small = (x.double() * 2.0 ** -50).to(x.dtype)  # exact; beside the squares eps is nothing
        _, q, unit, _, t = R.norm(small, w, None, 1e-6, True)
        rms = 1.0 / np.sqrt(np.square(small.double().numpy()).mean(1))
        assert np.array_equal(got.q.cpu().numpy(), q)
        off = R.norm_bound(d)
        assert np.all(np.abs(got.scale.cpu().numpy() - unit * rms) <= off * unit * rms)
        want = t * rms[:, None]
        assert np.all(np.abs(got.y.double().cpu().numpy() - want) <= np.abs(want) * (R.half_step(dtype) + 2 * off) + R.least(dtype))


@pytest.mark.parametrize("dtype,d", [("bf16", 2064), ("f32", 2064), ("f16", 6160), ("bf16", 16384)])
def test_norm_in_place_by_256_threads_to_a_row(dtype, d):
    rng = np.random.default_rng(d)
    x, r = rows_of(rng, 7, d, dtype), rows_of(rng, 7, d, dtype)
    weight = rows_of(rng, 1, d, dtype)[0].cuda()
    want = st.st_norm_rows(x.cuda(), weight, r.cuda())
    for place in ("x", "residual"):
        a, b = x.cuda(), r.cuda()
        got = st.st_norm_rows(a, weight, b, total=a if place == "x" else b)
        assert torch.equal(got.total, want.total) and torch.equal(got.q, want.q) and torch.equal(got.scale, want.scale)


# ---------------------------------------------------------------- values behind the last of k
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rank", [8, 24, 40, 128])
def test_infinite_adapter_at_the_last_values_of_k(rank, dtype):
    """A row's bits do not go by the number of rows beside it, where its adapter holds an infinity among the last values of k either."""
    say(f"[layer] infinity at the last values of k, rank {rank}, {dtype}")
    rng = np.random.default_rng(rank)
    k, n, rows = 80, 32, 2100
    x = integers(rng, rows, k).abs().clamp(1, 127)
    args = [x, torch.full((rows,), 2.0 ** -6), integers(rng, n, k), torch.full((n,), 2.0 ** -8)]
    a = torch.from_numpy(rng.normal(0, 1, (3, rank, k)).astype(np.float32)).to(R.TYPES[dtype])
    a[0, 0, 64], a[1, rank - 1, 71], a[2, 3, 72] = float("inf"), float("-inf"), float("inf")
    b = torch.from_numpy(rng.uniform(0.5, 1, (3, n, rank)).astype(np.float32)).to(R.TYPES[dtype])
    of = torch.from_numpy((np.arange(rows) % 3).astype(np.int32))
    got = call((*args, a, b, torch.ones(3), of))
    for m in (1, 20, 100, 500):
        few = call((args[0][:m], args[1][:m], *args[2:], a, b, torch.ones(3), of[:m]))
        assert torch.equal(few.view(torch.int16), got[:m].view(torch.int16))
    sign = torch.tensor([1.0, -1.0, 1.0], device="cuda")[of.cuda().long()]
    assert (got.float() == sign[:, None] * float("inf")).all()


# ---------------------------------------------------------------- positions far from the first
@pytest.mark.parametrize("inverse", [False, True])
def test_rotation_of_far_positions(inverse):
    """Sines and cosines off by 2^-22, and by 1.3 * 2^-52 of the angle, of which there are up to 2^33.6; angles reduced here in 200 bits."""
    say("[layer] rotation of far positions")
    rng = np.random.default_rng(17)
    n, d, pairs = 96, 64, 32
    pos = np.concatenate([rng.integers(-2 ** 31, 2 ** 31, n - 34), [2 ** 31 - 1, -2 ** 31], rng.integers(0, 2000, 32)]).astype(np.int32)
    freqs = np.concatenate([rng.uniform(np.pi, 2 * np.pi, 12), 2 * np.pi / 60 * (60 / 3.2e8) ** (np.arange(20) / 20)])
    pi = Fraction(314159265358979323846264338327950288419716939937510582097494459, 10 ** 62)
    angle = np.array([[float(a - 2 * pi * round(a / (2 * pi))) for a in (Fraction(int(p)) * Fraction(f) for f in freqs)] for p in pos])
    off = 2.0 ** -22 + 1.3 * 2.0 ** -52 * np.abs(pos.astype(np.float64)[:, None] * freqs)
    x = torch.from_numpy(rng.normal(0, 2, (n, 2, d)).astype(np.float32)).half()
    x[:, 0, pairs:] = 0  # cosines and sines by themselves
    got = st.st_rotate(x.cuda(), None, torch.from_numpy(pos[None]).cuda(), torch.from_numpy(freqs).cuda(), (pairs,), inverse=inverse)[0].double().cpu().numpy()
    cos, sin, off = np.cos(angle)[:, None], np.sin(angle)[:, None] * (-1 if inverse else 1), off[:, None]
    f = x.double().numpy()
    one, two = f[..., :pairs], f[..., pairs:]
    for out, want in ((got[..., :pairs], one * cos - two * sin), (got[..., pairs:], one * sin + two * cos)):
        bound = (np.abs(one) + np.abs(two)) * (off + 3 * R.F32)
        bound = bound + R.half_step("f16") * (np.abs(want) + bound) + R.least("f16")
        assert np.all(np.abs(out - want) <= bound), (np.abs(out - want) - bound).max()
