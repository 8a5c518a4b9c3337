"""Plain implementation, in 64 bits, of the operators of a layer around the cached histories (silvertorch.h), each with the
bound its outputs keep.  Roundings: a value rounded to a type is off by half a step at most, eps / 2 of it."""
import numpy as np
import torch

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
F32 = 2.0 ** -24  # half a step of fp32


def half_step(dtype):
    return torch.finfo(TYPES[dtype]).eps / 2


def least(dtype):
    """Half a step of the smallest numbers of the type."""
    return torch.finfo(TYPES[dtype]).smallest_normal * half_step(dtype) * 2


def norm(x, weight, residual, eps, normalise):
    """The sum (in x's type), integers, unit (fp32), and 1 / sqrt of the mean in 64 bits, row by row."""
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    f = h.float().numpy()
    t = f if weight is None else f * weight.float().numpy()  # fp32: one rounding
    unit = np.abs(t).max(1) / np.float32(127.0)
    with np.errstate(all="ignore"):
        q = np.where(unit[:, None] > 0, np.clip(np.rint(t / unit[:, None]), -127, 127), 0.0)
    mean = np.square(h.double().numpy()).mean(1)
    rms = 1.0 / np.sqrt(mean + np.float64(np.float32(eps))) if normalise else np.ones(len(t))
    return h, q.astype(np.int8), unit.astype(np.float64), rms, t.astype(np.float64)


def norm_bound(d):
    """Relative error of 1 / sqrt(mean + eps): the mean's sum of squares (all positive) goes through at most d / 16 + 24 additions of a
    chain, of which a root takes half; then the mean's division, the sum with eps, root, inverse, one product."""
    return ((d / 16 + 24 + 3) / 2 + 4) * F32


def project(x, x_scale, w, w_scale, a=None, b=None, alpha=None, adapter_of=None, dtype="bf16"):
    """Outputs and their bound."""
    x64, xs = x.double().numpy(), x_scale.double().numpy()[:, None]
    base = x64 @ w.double().numpy().T * xs * w_scale.double().numpy()
    out, bound = base.copy(), 4 * F32 * np.abs(base)  # conversion, two products
    if a is not None:
        half = half_step(dtype)
        k, rank = a.shape[2], a.shape[1]
        for t, i in enumerate(adapter_of.tolist()):
            if not 0 <= i < a.shape[0]:
                continue
            a64, b64, f = a[i].double().numpy(), b[i].double().numpy(), float(alpha[i]) * xs[t, 0]
            inner = (a64 @ x64[t]) * f
            # fp32 sums of k products in any order, two products; rounding to the type, of which fp16 ends 2^-24 below the largest
            off = (k + 8) * F32 * (np.abs(a64) @ np.abs(x64[t])) * abs(f) + half * np.abs(inner)
            off += (2.0 ** -24 if dtype == "f16" else 0.0) * np.abs(inner).max()
            size = np.abs(b64) @ np.abs(inner)
            out[t] += b64 @ inner
            bound[t] += np.abs(b64) @ off * (1 + half) + (rank + 8) * F32 * (size + np.abs(base[t]))
    return out, bound + half_step(dtype) * (np.abs(out) + bound) + least(dtype)


def rotate(rows, positions, freqs, sections, interleaved, inverse, dtype):
    """Rotated rows and their bound: cos and sin off by 2^-20, two products and a sum in fp32, one rounding."""
    axis = np.repeat(np.arange(len(sections)), sections)
    angle = positions.double().numpy()[axis].T * freqs.double().numpy()
    cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None] * (-1 if inverse else 1)
    pairs = len(axis)
    x = rows.double().numpy()
    i, j = (np.arange(0, 2 * pairs, 2), np.arange(1, 2 * pairs, 2)) if interleaved else (np.arange(pairs), np.arange(pairs, 2 * pairs))
    out, bound = x.copy(), np.zeros_like(x)
    out[..., i], out[..., j] = x[..., i] * cos - x[..., j] * sin, x[..., i] * sin + x[..., j] * cos
    size = np.abs(x[..., i]) + np.abs(x[..., j])
    for c in (i, j):
        bound[..., c] = size * (2.0 ** -20 + 3 * F32) + half_step(dtype) * np.abs(out[..., c]) * (1 + 2.0 ** -10) + least(dtype)
    return out, bound
