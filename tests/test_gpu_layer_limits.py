"""The operators of a layer around the cached histories where their numbers end: inner values that cancel.
Bounds: layer_reference, or derived here."""
import numpy as np
import pytest
import torch

from paper_2511_14881_amd import binding as st
from tests import layer_reference as R
from tests.test_gpu_layer import call, integers, say

pytestmark = pytest.mark.gpu

# rows that take each route at k = 64 to 272 and few columns: one launch, few rows, several workgroups of them, tiles with and without an order
ROUTES = [2, 20, 100, 600, 2100]


# ---------------------------------------------------------------- inner values that cancel
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n_rows", ROUTES)
def test_projection_of_inner_values_that_cancel(n_rows, dtype):
    """Ranks in pairs of nearly the same inner value, with opposite signs behind them: what is left of a pair is some 2^-8 of either.  All sums
    before the rounding to two 16-bit halves are of integers below 2^24, with factors that are powers of two, and so exact; the halves leave
    half a step of half a step (and fp16's smallest numbers, whose half step is 2^-25 beside a row's largest value in [1, 2))."""
    say(f"[layer] cancelling inner values, {n_rows} rows, {dtype}")
    rng = np.random.default_rng(n_rows)
    k, n, rank, count = 64, 48, 8 if n_rows == 2 else 24, 6
    x = integers(rng, n_rows, k)
    a = rng.integers(-64, 65, (count, rank, k))
    a[:, 1::2] = np.clip(a[:, 0::2] + rng.integers(-1, 2, (count, rank // 2, k)) * (rng.random((count, rank // 2, k)) < 0.1), -64, 64)
    b = rng.integers(-64, 65, (count, n, rank))
    b[:, :, 1::2] = -b[:, :, 0::2]
    of = rng.integers(-1, count, n_rows)
    half = R.half_step(dtype)
    size = -10  # outputs of fp16's range
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
