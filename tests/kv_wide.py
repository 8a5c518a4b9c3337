"""The plain implementation of attention over cached histories (kv_reference) for many rows and long histories: the same
definition in 64 bits, a sequence and head at a time, with what error bounds need."""
import copy

import numpy as np

from tests import kv_reference as R


def visible(host, s, off, causal, mask):
    """Truth values [tokens of sequence s, length]."""
    n, count = host.lens[s], off[s + 1] - off[s]
    t = np.arange(n)
    ok = t < (n - (count - 1 - np.arange(count))[:, None] if causal else n)
    ok = np.broadcast_to(ok, (count, n))
    if mask is not None and n:
        words = mask[off[s]:off[s + 1]][:, t // 64]
        ok = ok & ((words >> (t % 64).astype(np.uint64)) & np.uint64(1) != 0)
    return ok


def attend(host, q, scale, causal=True, offsets=None, mask=None, blocks=None, mass=None, decay=1.0):
    """(out, lse, mass, reach, value): kv_reference.attend's, and value [n_tok, heads]: the largest magnitude that the row's visible
    blocks can hold, 127 of the largest of their scales."""
    q64 = R.to_float(q)
    n_tok, n_qh, d = q64.shape
    group = n_qh // host.heads
    out, lse = np.zeros((n_tok, n_qh, d)), np.full((n_tok, n_qh), -np.inf)
    reach, value = np.zeros((n_tok, n_qh)), np.zeros((n_tok, n_qh))
    total = np.zeros((len(host.lens), host.heads, host.max_blocks)) if mass is None else mass.astype(np.float64) * np.float32(decay)
    off = R.offsets_of(len(host.lens), n_tok, offsets)
    for s, n in enumerate(host.lens):
        held = -(-n // R.BLOCK)
        total[s, :, held:] = 0.0
        rows = slice(off[s], off[s + 1])
        if n == 0 or off[s + 1] == off[s]:
            continue
        seen = visible(host, s, off, causal, mask)
        at = np.arange(n) // R.BLOCK
        for h in range(host.heads):
            k, v = host.rows(s, h)
            ok = seen
            if blocks is not None:
                listed = np.zeros((len(seen), held + 1), bool)
                pick = blocks[rows, h]
                np.put_along_axis(listed, np.where((pick >= 0) & (pick < held), pick, held), True, 1)
                ok = ok & listed[:, :held][:, at]
            some = ok.any(1)
            scales = np.abs(host.vs[host.tables[s, :held], h].astype(np.float64))
            for g in range(h * group, (h + 1) * group):
                x = np.where(ok, q64[rows, g] @ k.T * scale, -np.inf)
                top = np.where(some, x.max(1), 0.0)[:, None]
                e = np.exp(x - top)
                total_e = np.where(some, e.sum(1), 1.0)[:, None]
                p = e / total_e
                out[rows, g] = p @ v
                lse[rows, g] = np.where(some, (top + np.log(total_e))[:, 0], -np.inf)
                reach[rows, g] = np.where(ok, np.abs(q64[rows, g]) @ np.abs(k).T, 0.0).max(1) * abs(scale)
                value[rows, g] = 127.0 * np.where(ok, scales[at], 0.0).max(1)
                total[s, h, :held] += np.add.reduceat(p.sum(0), np.arange(0, n, R.BLOCK))
    return out, lse, total, reach, value


def error(host, want, reach, value, dtype, tokens=None):
    """Bound of an output's error, element by element (test_gpu_kv's, with the row's own largest value)."""
    T = max(host.lens) if tokens is None else tokens
    rel = (2 * (host.d + 8) * reach * 2.0 ** -24 + 2.0 ** -12 + (T / 16 + 64) * 2.0 ** -23)[..., None]
    half = 2.0 ** -8 * np.abs(want) + 2.0 ** -133 if dtype == "bf16" else 2.0 ** -11 * np.abs(want) + 2.0 ** -24
    return rel * value[..., None] + half


def check(got, want, bound):
    got = got.float().cpu().numpy().astype(np.float64)
    assert np.isfinite(got).all()
    over = np.abs(got - want) - bound
    at = np.unravel_index(over.argmax(), over.shape)
    assert over[at] <= 0, f"{got[at]} where {want[at]} is right, off by {abs(got[at] - want[at])} of {bound[at]} at {at}"


def lse_error(host, want_lse, reach):
    return (2 * (host.d + 8) * reach + max(host.lens) / 16 + 64 + 4 * np.abs(np.where(np.isfinite(want_lse), want_lse, 0))) * 2.0 ** -23


def shared(host, lens):
    """The host's only sequence as one for each of lens, all on its pages."""
    nb = host.tables.shape[1]
    held = -(-np.asarray(lens) // R.BLOCK)
    host.tables = np.where(np.arange(nb) < held[:, None], host.tables, -1).astype(np.int32)
    host.lens = list(lens)
    return host


def part(host, seqs):
    """The host with these of its sequences alone."""
    some = copy.copy(host)
    some.tables, some.lens = host.tables[seqs], [host.lens[s] for s in seqs]
    return some
