"""Plain implementation, in 64 bits and loops, of the operators on cached histories (silvertorch.h), and caches to
try them on: pages in random order, garbage wherever no token lies."""
import math

import numpy as np
import torch

BLOCK = 64


def slot(t):
    bits = [(t >> i) & 1 for i in range(6)]
    return bits[3] << 5 | bits[2] << 4 | bits[5] << 3 | bits[4] << 2 | bits[1] << 1 | bits[0]


SLOTS = np.array([slot(t) for t in range(BLOCK)])


def to_float(x):
    return x.float().numpy().astype(np.float64)


class Host:
    """A cache and its sequences as numpy arrays, and as the tensors of a call."""

    def __init__(self, rng, lens, heads, d, spare=5, max_blocks=None):
        held = [-(-n // BLOCK) for n in lens]
        n_pages = sum(held) + spare
        self.lens, self.heads, self.d = list(lens), heads, d
        self.max_blocks = max_blocks or max(1, max(held))
        order = rng.permutation(n_pages)
        self.tables = np.full((len(lens), self.max_blocks), -1, np.int32)
        # what no token occupies is filled with the worst: extreme integers, scales that are not numbers
        self.k = rng.integers(0, 2, (n_pages, heads, BLOCK, d)).astype(np.int8) * 127
        self.v = rng.integers(0, 2, (n_pages, heads, BLOCK, d)).astype(np.int8) * -128
        self.ks = np.full((n_pages, heads), np.nan, np.float32)
        self.vs = np.full((n_pages, heads), np.nan, np.float32)
        self.bounds = rng.integers(-128, 128, (n_pages, heads, 2, d)).astype(np.int8)
        at = 0
        for s, n in enumerate(lens):
            for b in range(held[s]):
                p = order[at]
                at += 1
                self.tables[s, b] = p
                m = min(BLOCK, n - b * BLOCK)
                self.k[p, :, :m] = np.clip(np.rint(rng.normal(0, 40, (heads, m, d))), -127, 127)
                self.v[p, :, :m] = np.clip(np.rint(rng.normal(0, 40, (heads, m, d))), -127, 127)
                self.ks[p] = rng.uniform(0.005, 0.06, heads)
                self.vs[p] = rng.uniform(0.001, 0.1, heads)
                self.bounds[p, :, 0] = self.k[p, :, :m].max(1)
                self.bounds[p, :, 1] = self.k[p, :, :m].min(1)

    def cache(self, st):
        v = np.empty((*self.v.shape[:2], self.d, BLOCK), np.int8)
        v[..., SLOTS] = self.v.swapaxes(2, 3)
        return st.KvCache(*(torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (self.k, v, self.ks, self.vs, self.bounds)))

    def batch(self, st, n_tok, offsets=None, **kw):
        off = None if offsets is None else torch.tensor(offsets, dtype=torch.int32).cuda()
        return st.KvBatch(torch.from_numpy(self.tables).cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda(), n_tok,
                          offsets=off, **kw)

    def rows(self, s, h):
        """Keys and values of a sequence and head, in 64 bits."""
        p = self.tables[s, : -(-self.lens[s] // BLOCK)]
        n = self.lens[s]
        k = (self.k[p, h].astype(np.float64) * self.ks[p, h].astype(np.float64)[:, None, None]).reshape(-1, self.d)[:n]
        v = (self.v[p, h].astype(np.float64) * self.vs[p, h].astype(np.float64)[:, None, None]).reshape(-1, self.d)[:n]
        return k, v


def offsets_of(n_seq, n_tok, offsets):
    return offsets if offsets is not None else [i * (n_tok // n_seq) for i in range(n_seq + 1)]


def sees(host, s, i, count, causal, mask_row):
    """Truth values [length]: what token i of `count` sees."""
    n = host.lens[s]
    t = np.arange(n)
    ok = t < (n - (count - 1 - i) if causal else n)
    if mask_row is not None:
        ok &= (mask_row[t // 64] >> (t % 64).astype(np.uint64)) & np.uint64(1) != 0
    return ok


def attend(host, q, scale, causal, offsets=None, mask=None, blocks=None, mass=None, decay=1.0):
    """(out, lse, mass, reach): reach [n_tok, heads] is the largest sum of |q_c k_c| * scale of a row, for error bounds."""
    q64 = to_float(q)
    n_tok, n_qh, d = q64.shape
    group = n_qh // host.heads
    out, lse = np.zeros((n_tok, n_qh, d)), np.full((n_tok, n_qh), -np.inf)
    reach = np.zeros((n_tok, n_qh))
    total = np.zeros((len(host.lens), host.heads, host.max_blocks)) if mass is None else mass.astype(np.float64) * np.float32(decay)
    off = offsets_of(len(host.lens), n_tok, offsets)
    for s, n in enumerate(host.lens):
        total[s, :, -(-n // BLOCK):] = 0.0
        for tok in range(off[s], off[s + 1]):
            ok0 = sees(host, s, tok - off[s], off[s + 1] - off[s], causal, None if mask is None else mask[tok])
            for h in range(host.heads):
                k, v = host.rows(s, h)
                ok = ok0
                if blocks is not None:
                    ok = ok & np.isin(np.arange(n) // BLOCK, blocks[tok, h])
                if not ok.any():
                    continue
                for g in range(h * group, (h + 1) * group):
                    x = (k[ok] @ q64[tok, g]) * scale
                    top = x.max()
                    e = np.exp(x - top)
                    p = e / e.sum()
                    out[tok, g] = p @ v[ok]
                    lse[tok, g] = top + math.log(e.sum())
                    reach[tok, g] = (np.abs(k[ok]) @ np.abs(q64[tok, g])).max() * abs(scale)
                    total[s, h] += np.bincount(np.nonzero(ok)[0] // BLOCK, weights=p, minlength=host.max_blocks)
    return out, lse, total, reach


def order_key(scores, index):
    return sorted(index, key=lambda b: (-scores[b], b))


def select(host, q, n_sel, causal, sink, recent, offsets=None, mask=None):
    q32 = q.float().numpy()
    n_tok, n_qh, d = q32.shape
    group = n_qh // host.heads
    out = np.full((n_tok, host.heads, n_sel), -1, np.int32)
    off = offsets_of(len(host.lens), n_tok, offsets)
    for s, n in enumerate(host.lens):
        pages = host.tables[s, : -(-n // BLOCK)]
        for tok in range(off[s], off[s + 1]):
            i, count = tok - off[s], off[s + 1] - off[s]
            ok = sees(host, s, i, count, causal, None if mask is None else mask[tok])
            able = [b for b in range(len(pages)) if ok[b * BLOCK:(b + 1) * BLOCK].any()]
            n_seen = -(-max(0, n - (count - 1 - i) if causal else n) // BLOCK)
            for h in range(host.heads):
                u = np.zeros(2 * d, np.float32)
                for g in range(h * group, (h + 1) * group):
                    u = u + np.concatenate([np.maximum(q32[tok, g], 0), np.minimum(q32[tok, g], 0)])
                unit = np.abs(u).max() / np.float32(127)
                u8 = np.clip(np.rint(u / unit), -127, 127).astype(np.int64) if unit > 0 else np.zeros(2 * d, np.int64)
                dots = host.bounds[pages, h].reshape(len(pages), 2 * d).astype(np.int64) @ u8
                score = dots.astype(np.float32) * host.ks[pages, h]
                always = [b for b in able if b < sink or b >= n_seen - recent]
                best = order_key(score, [b for b in able if b not in always])
                chosen = sorted((always + best)[:n_sel])
                out[tok, h, : len(chosen)] = chosen
    return out


def evict(tables, lens, mass, budget, sink, recent):
    n_seq, nb = tables.shape
    out = np.full_like(tables, -1), np.zeros(n_seq, np.int32), np.zeros_like(mass), np.full_like(tables, -1), np.zeros(n_seq, np.int32)
    for s, n in enumerate(lens):
        held = -(-n // BLOCK)
        score = mass[s].max(0)
        always = [b for b in range(held) if b < sink or b >= held - recent]
        keep = sorted((always + order_key(score, [b for b in range(held) if b not in always]))[:budget])
        gone = [b for b in range(held) if b not in keep]
        out[0][s, : len(keep)] = tables[s, keep]
        out[1][s] = n - BLOCK * len(gone)
        out[2][s, :, : len(keep)] = mass[s][:, keep]
        out[3][s, : len(gone)] = tables[s, gone]
        out[4][s] = len(gone)
    return out


def append(host, k_new, v_new, offsets=None):
    """Moves host to the state after the call (its lengths are those after it)."""
    n_tok = k_new.shape[0]
    off = offsets_of(len(host.lens), n_tok, offsets)
    for s, n in enumerate(host.lens):
        count = off[s + 1] - off[s]
        begin = n - count
        for b in range(max(begin, 0) // BLOCK, -(-n // BLOCK)):
            p = host.tables[s, b]
            if p < 0 or p >= len(host.k) or count == 0:
                continue
            t0, t1 = max(begin - b * BLOCK, 0), min(n - b * BLOCK, BLOCK)
            r0 = off[s] + b * BLOCK - begin
            for new, held, scale in ((k_new, host.k, host.ks), (v_new, host.v, host.vs)):
                x = new[r0 + t0: r0 + t1].float().numpy()  # [tokens, heads, d]
                for h in range(host.heads):
                    old = scale[p, h] if t0 > 0 else np.float32(0)
                    grown = max(old, np.abs(x[:, h]).max() / np.float32(127))
                    ratio = np.float32(old / grown) if grown > 0 else np.float32(0)
                    held[p, h, :t0] = np.rint(held[p, h, :t0].astype(np.float32) * ratio)
                    held[p, h, t0:t1] = np.clip(np.rint(x[:, h] / grown), -127, 127) if grown > 0 else 0
                    scale[p, h] = grown
            host.bounds[p, :, 0] = host.k[p, :, :t1].max(1)
            host.bounds[p, :, 1] = host.k[p, :, :t1].min(1)
