#!/usr/bin/env python3
"""Users' event histories beside the index: a store of cached keys and values (``HistoryStore``), and a serving loop that
runs it with the search as they would be used together.

    python -m paper_2511_14881_amd.history [--items 200000] [--users 64] [--events 3000] [--steps 8] [--layer]

Each step of the loop searches the index for every user (``st_search``), lets the retrieved candidates attend to the
user's history, whole or in the blocks each candidate selects, ranks them by the attended interest, appends the
winner to the history as a new event, lets the newest event attend and so accumulate what weight the blocks draw, and
cuts histories that outgrow their budget.  The events' keys are item embeddings, their values the embeddings again: a
stand-in for the trained projections of a ranking model.  With --layer they go through a layer with such projections
(``HistoryLayer``, its weights random, an adapter for each of three markets, positions by index and time), which also
makes the next search's queries and each user's alternative: a fork of the history that takes the second best event.  Prints one JSON line.
"""
from __future__ import annotations

import argparse
import json
import sys
import time

import numpy as np
import torch

from paper_2511_14881_amd import binding as st


class HistoryStore:
    """Pages of one ``KvCache`` dealt out to users.  Tables and lengths are kept on the host, where pages are
    handed out and taken back, and copied to the device for a call; the blocks' accumulated weights stay there.
    Histories may share pages (``fork``): a page is written by an append only where one history has it, and comes free with the last."""

    def __init__(self, n_users: int, n_pages: int, n_heads: int, d: int, max_blocks: int):
        self.cache = st.KvCache.empty(n_pages, n_heads, d)
        self.max_blocks = max_blocks
        self.tables = np.full((n_users, max_blocks), -1, np.int32)
        self.lengths = np.zeros(n_users, np.int32)
        self.mass = torch.zeros((n_users, n_heads, max_blocks), dtype=torch.float32, device="cuda")
        self.free = list(range(n_pages - 1, -1, -1))
        self.shares = np.zeros(n_pages, np.int32)  # histories that hold a page
        self.forked = False  # whether there may be more than one to a page

    def _known(self, users, once: bool = False) -> np.ndarray:
        """The users as an array of indices.  once: none may be named twice, since the call writes to their histories."""
        users = np.asarray(users)
        if users.ndim != 1 or (users.size and users.dtype.kind not in "iu"):
            raise ValueError("users must be whole numbers in a row")
        if users.size and (users.min() < 0 or users.max() >= len(self.lengths)):
            raise ValueError(f"users must be in [0, {len(self.lengths)})")
        if once and len(np.unique(users)) != len(users):
            raise ValueError("a user is named twice: join what belongs to one history")
        return users.astype(np.int64)  # (an empty list comes as floats)

    @staticmethod
    def _counts(users, counts) -> np.ndarray:
        counts = np.ones(len(users), np.int64) if counts is None else np.asarray(counts, dtype=np.int64)
        if counts.shape != (len(users),) or (counts.size and counts.min() < 0):
            raise ValueError(f"counts must be {len(users)} numbers, none below 0")
        return counts

    @staticmethod
    def _view(tables, lengths, counts) -> st.KvBatch:
        offsets = None
        if counts.size and counts.min() != counts.max():
            offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda()
        return st.KvBatch(torch.from_numpy(tables).cuda(), torch.from_numpy(lengths).cuda(), int(counts.sum()), offsets=offsets,
                          max_tok=int(counts.max()) if counts.size else 0, max_len=int(lengths.max()) if lengths.size else 0)

    def batch(self, users, counts) -> st.KvBatch:
        """The call's view of these users, counts[i] tokens of users[i] in it."""
        return self._view(self.tables[users], self.lengths[users], self._counts(users, counts))

    def append(self, users, k, v, counts=None) -> None:
        """Events k, v [sum of counts, heads, d] behind the users' histories (one each if counts is not given).
        Each user once.  A call that is refused leaves the store as it was."""
        users = self._known(users, once=True)
        counts = self._counts(users, counts)
        if len(users) == 0:
            return
        tables, lengths = self.tables[users], self.lengths[users]
        have, need = -(-lengths // st.ST_KV_BLOCK), -(-(lengths + counts) // st.ST_KV_BLOCK)
        if need.size and need.max() > self.max_blocks:
            raise ValueError(f"a history would hold {need.max()} blocks of at most {self.max_blocks}: evict first")
        # where the block that the first event goes to is shared, the history gets a copy of its own; the last holder keeps the page
        left, copied = {}, []  # of such pages, the histories that still hold them
        if self.forked:
            tails = tables[np.arange(len(users)), np.maximum(have - 1, 0)]
            for i in np.flatnonzero((lengths % st.ST_KV_BLOCK > 0) & (counts > 0) & (self.shares[tails] > 1)):
                holders = left.get(tails[i], self.shares[tails[i]])
                if holders > 1:
                    left[tails[i]] = holders - 1
                    copied.append((i, tails[i]))
        taken = int((need - have).sum()) + len(copied)
        if taken > len(self.free):
            raise ValueError(f"{taken} pages are needed, {len(self.free)} are free: evict first")
        new = self.free[len(self.free) - taken:][::-1]
        pages = iter(new)
        for row, a, b in zip(tables, have, need):
            for block in range(a, b):
                row[block] = next(pages)
        if copied:
            for i, _ in copied:
                tables[i, have[i] - 1] = next(pages)
            self._copy(self.cache, self.cache, [page for _, page in copied], [tables[i, have[i] - 1] for i, _ in copied])
        lengths = (lengths + counts).astype(np.int32)
        st.st_kv_append(self.cache, self._view(tables, lengths, counts), k, v)
        self.tables[users], self.lengths[users] = tables, lengths
        if new:
            self.shares[new] = 1
        for page, holders in left.items():
            self.shares[page] = holders
        del self.free[len(self.free) - taken:]

    def attend(self, users, q, counts, n_sel: int = 0, sink: int = 0, recent: int = 0, causal: bool = False, track: bool = False,
               decay: float = 1.0, mask=None) -> torch.Tensor:
        """Outputs like q [sum of counts, q_heads, d] over the users' histories, or over the n_sel blocks that each row
        selects.  track: the blocks' accumulated weights decay and take on what this call gave them (each user once)."""
        users = self._known(users, once=track)
        counts = self._counts(users, counts)
        if len(users) == 0:
            return torch.empty_like(q)
        batch = self.batch(users, counts)
        blocks = None
        if n_sel:
            blocks = st.st_kv_select(self.cache, batch, q, n_sel, causal=causal, mask=mask, sink=sink, recent=recent)
        if not track:
            return st.st_kv_attend(self.cache, batch, q, causal=causal, mask=mask, blocks=blocks)
        rows = torch.from_numpy(users).cuda()
        mass = self.mass[rows]
        out = st.st_kv_attend(self.cache, batch, q, causal=causal, mask=mask, blocks=blocks, mass=mass, decay=decay, mass_out=mass)
        self.mass[rows] = mass
        return out

    def evict(self, users, budget: int, sink: int = 0, recent: int = 1) -> int:
        """Cuts the users' histories to at most budget blocks; returns how many pages came free.  Each user once."""
        users = self._known(users, once=True)
        if len(users) == 0:
            return 0
        rows = torch.from_numpy(users).cuda()
        tables, lengths, mass, freed, n_freed = st.st_kv_evict(self.batch(users, np.zeros(len(users))), self.mass[rows], budget,
                                                               sink=sink, recent=recent)
        self.tables[users], self.lengths[users] = tables.cpu().numpy(), lengths.cpu().numpy()
        self.mass[rows] = mass
        pages, count = freed.cpu().numpy(), n_freed.cpu().numpy()
        return sum(self._give_back(pages[i, :n]) for i, n in enumerate(count))

    def _give_back(self, pages) -> int:
        """One history less holds the pages; returns how many came free."""
        before = len(self.free)
        for page in pages.tolist():
            self.shares[page] -= 1
            if self.shares[page] == 0:
                self.free.append(page)
        return len(self.free) - before

    @staticmethod
    def _copy(from_cache, to_cache, src, dst) -> None:
        lists = torch.from_numpy(np.array([src, dst], np.int32)).cuda()
        st.st_kv_copy(from_cache, to_cache, lists[0], lists[1])

    def fork(self, users, to) -> None:
        """Each of the users `to`, whose histories are empty, gets the history of the user beside it, with its blocks' weights.  The
        pages are shared until one of the histories appends to a page that is not full."""
        users, to = self._known(users), self._known(to, once=True)
        if users.shape != to.shape:
            raise ValueError("as many users to fork as histories to fill")
        if self.lengths[to].any():
            raise ValueError("a history that is not empty would be lost: release it first")
        if len(users) == 0:
            return
        self.tables[to], self.lengths[to] = self.tables[users], self.lengths[users]
        held = self.tables[to]
        np.add.at(self.shares, held[held >= 0], 1)
        self.forked = True
        self.mass[torch.from_numpy(to).cuda()] = self.mass[torch.from_numpy(users).cuda()]

    def release(self, users) -> int:
        """The users' histories end; returns how many pages came free.  Each user once."""
        users = self._known(users, once=True)
        if len(users) == 0:
            return 0
        freed = sum(self._give_back(row[row >= 0]) for row in self.tables[users])
        self.tables[users], self.lengths[users] = -1, 0
        self.mass[torch.from_numpy(users).cuda()] = 0.0
        return freed

    def compact(self) -> int:
        """Moves what lies behind the first pages of the cache, as many as are in use, into the free ones among them; returns how
        many pages moved.  Batches that a program holds name the pages as they were."""
        used = np.flatnonzero(self.shares)
        src = used[used >= len(used)]
        dst = np.flatnonzero(self.shares[: len(used)] == 0)
        if len(src):
            self._copy(self.cache, self.cache, src, dst)
            place = np.arange(len(self.shares), dtype=np.int32)
            place[src] = dst
            self._moved(place, len(self.shares))
        return len(src)

    def resize(self, n_pages: int) -> None:
        """A cache of n_pages pages, at least those in use, in place of the one so far; the pages in use are its first ones.  Batches and
        buffers that a program holds of the cache so far are not of the new one."""
        used = np.flatnonzero(self.shares)
        if n_pages < max(1, len(used)):
            raise ValueError(f"{len(used)} pages are in use, {n_pages} are too few")
        cache = st.KvCache.empty(n_pages, self.cache.n_heads, self.cache.d)
        if len(used):
            self._copy(self.cache, cache, used, np.arange(len(used)))
        place = np.full(len(self.shares), -1, np.int32)
        place[used] = np.arange(len(used))
        self._moved(place, n_pages)
        self.cache = cache

    def _moved(self, place, n_pages: int) -> None:
        """Page p is now page place[p], of n_pages."""
        used = np.flatnonzero(self.shares)
        shares = np.zeros(n_pages, np.int32)
        shares[place[used]] = self.shares[used]
        held = self.tables >= 0
        self.tables[held] = place[self.tables[held]]
        self.shares = shares
        self.free = [int(p) for p in np.flatnonzero(shares == 0)[::-1]]


def _loop_with_layer(args, cfg, w, bloom):
    from paper_2511_14881_amd.layer import HistoryLayer

    gen = torch.Generator(device="cuda").manual_seed(cfg.seed)
    heads, kv_heads, d, markets, rank, width, n_users, K = 4, 2, 64, 3, 16, cfg.d, args.users, cfg.top_k

    def normal(*shape, size=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * size).to(torch.bfloat16)

    def adapters(n, k):
        return normal(markets, rank, k, size=k ** -0.5), normal(markets, n, rank, size=0.1), torch.full((markets,), 0.5, device="cuda")

    n_qkv = (heads + 2 * kv_heads) * d
    # an index, and a time in seconds with periods from a minute to a year
    freqs = torch.cat([10000.0 ** (-torch.arange(16) / 16), 2 * np.pi / 60 * (60 / 3.2e7) ** (torch.arange(16) / 16)]).double().cuda()
    layer = HistoryLayer(heads, kv_heads, d, torch.ones(width, dtype=torch.bfloat16, device="cuda"), normal(n_qkv, width, size=width ** -0.5),
                         normal(width, heads * d, size=(heads * d) ** -0.5), (16, 16), freqs, adapters(n_qkv, width),
                         adapters(width, heads * d))
    embedding = (w.items.float() * w.item_scale[:, None]).to(torch.bfloat16)
    users, blocks = np.arange(n_users), args.events // st.ST_KV_BLOCK + 4
    store = HistoryStore(2 * n_users, 2 * n_users * blocks, kv_heads, d, max_blocks=blocks)  # and a place for each user's alternative
    market = torch.arange(n_users, dtype=torch.int32, device="cuda") % markets
    counts = np.maximum(1, args.events - np.arange(n_users) * args.events // (2 * n_users))
    repeat = torch.from_numpy(counts).cuda()
    index = torch.cat([torch.arange(n) for n in counts]).int().cuda()
    seen = torch.randint(0, cfg.n_items, (int(counts.sum()),), generator=gen, device="cuda")
    layer.take_in(store, users, embedding[seen], torch.stack([index, 1_700_000_000 + 60 * index]), counts, market.repeat_interleave(repeat))
    state = embedding[seen[repeat.cumsum(0) - 1]]
    at, freed, begun = repeat.int(), 0, time.perf_counter()
    for step in range(args.steps):
        now = torch.stack([at, 1_700_000_000 + 60 * at])
        out, total = layer(store, users, state, now, tenants=market, track=True, decay=0.9)
        query = st.st_norm_rows(out, layer.norm, total)
        ids, _, _ = st.st_search(bloom, w.items, w.item_scale, query.q, query.scale, w.filt_ids, w.filt_offsets, K)[:3]
        rows = embedding[ids.clamp_min(0)].view(-1, width)
        interest, _ = layer(store, users, rows, now.repeat_interleave(K, 1), [K] * n_users, market.repeat_interleave(K), append=False,
                            n_sel=args.select if step % 2 else 0)
        rank_by = (interest.float() * rows.float()).sum(1).view(n_users, K).masked_fill(ids < 0, -float("inf"))
        best = ids.gather(1, rank_by.topk(min(2, K)).indices).clamp_min(0)
        # what each history would be with the second best event instead
        others = users + n_users
        freed += store.release(others)
        store.fork(users, others)
        other, _ = layer(store, others, embedding[best[:, -1]], now + 1, tenants=market)
        state, at = embedding[best[:, 0]], at + 1
        over = users[-(-store.lengths[:n_users] // st.ST_KV_BLOCK) > args.budget]
        freed += store.evict(over, args.budget, sink=1, recent=2)
    freed += store.release(users + n_users)
    moved = store.compact()
    store.resize(max(1, int((store.shares > 0).sum())))
    torch.cuda.synchronize()
    spent = time.perf_counter() - begun
    print(json.dumps({"users": n_users, "items": cfg.n_items, "candidates": K, "steps": args.steps, "ms_per_step": spent * 1e3 / args.steps,
                      "pages_freed": freed, "pages_moved": moved, "pages": store.cache.n_pages, "longest": int(store.lengths.max()),
                      "finite": bool(torch.isfinite(rank_by[ids >= 0]).all() and torch.isfinite(other.float()).all())}))
    bloom.free()


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--items", type=int, default=200_000)
    ap.add_argument("--users", type=int, default=64)
    ap.add_argument("--events", type=int, default=3000)
    ap.add_argument("--candidates", type=int, default=100)
    ap.add_argument("--select", type=int, default=8, help="blocks each candidate reads in every other step (0: always all)")
    ap.add_argument("--budget", type=int, default=40, help="blocks a history may hold")
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--layer", action="store_true", help="a layer with projections, adapters and positions in place of bare embeddings")
    args = ap.parse_args()
    from paper_2511_14881_amd import synth

    if not torch.cuda.is_available():
        print("history needs a GPU", file=sys.stderr)
        sys.exit(2)
    cfg = synth.scaled(synth.CONFIGS["mid"], args.items, batch=args.users, top_k=args.candidates)
    w = synth.make_workload(cfg, device="cuda")
    bloom = st.st_bloom_build(w.feat_offsets, w.feat_ids, cfg.n_items, cfg.m_bits, cfg.k_hashes)
    if args.layer:
        return _loop_with_layer(args, cfg, w, bloom)
    heads, d = 2, cfg.d // 2
    embedding = (w.items.float() * w.item_scale[:, None]).to(torch.bfloat16).view(cfg.n_items, heads, d)
    users = np.arange(args.users)
    store = HistoryStore(args.users, args.users * (args.events // st.ST_KV_BLOCK + 4), heads, d,
                         max_blocks=args.events // st.ST_KV_BLOCK + 4)
    gen = torch.Generator(device="cuda").manual_seed(cfg.seed)
    counts = np.maximum(1, args.events - np.arange(args.users) * args.events // (2 * args.users))
    seen = torch.randint(0, cfg.n_items, (int(counts.sum()),), generator=gen, device="cuda")
    store.append(users, embedding[seen], embedding[seen], counts)
    freed, begun = 0, time.perf_counter()
    for step in range(args.steps):
        ids, scores, count = st.st_search(bloom, w.items, w.item_scale, w.queries, w.query_scale, w.filt_ids, w.filt_offsets,
                                          cfg.top_k)
        rows = embedding[ids.clamp_min(0)].view(-1, heads, d)
        interest = store.attend(users, rows, [cfg.top_k] * args.users, n_sel=args.select if step % 2 else 0)
        rank = (interest.float() * rows.float()).sum((1, 2)).view(args.users, cfg.top_k)
        rank = rank.masked_fill(ids < 0, -float("inf"))
        best = ids.gather(1, rank.argmax(1, keepdim=True))[:, 0].clamp_min(0)
        event = embedding[best]
        store.append(users, event, event)
        store.attend(users, event, [1] * args.users, causal=True, track=True, decay=0.9)
        over = users[-(-store.lengths // st.ST_KV_BLOCK) > args.budget]
        freed += store.evict(over, args.budget, sink=1, recent=2)
    torch.cuda.synchronize()
    spent = time.perf_counter() - begun
    print(json.dumps({"users": args.users, "items": cfg.n_items, "candidates": cfg.top_k, "steps": args.steps,
                      "ms_per_step": spent * 1e3 / args.steps, "pages_freed": freed, "free_pages": len(store.free),
                      "longest": int(store.lengths.max()), "finite": bool(torch.isfinite(rank[ids >= 0]).all())}))
    bloom.free()


if __name__ == "__main__":
    main()
