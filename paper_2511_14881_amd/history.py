#!/usr/bin/env python3
"""Users' event histories beside the index: a store of cached keys and values (``HistoryStore``), and a serving loop that
runs it with the search as they would be used together.

    python -m paper_2511_14881_amd.history [--items 200000] [--users 64] [--events 3000] [--steps 8]

Each step of the loop searches the index for every user (``st_search``), lets the retrieved candidates attend to the
user's history, whole or in the blocks each candidate selects, ranks them by the attended interest, appends the
winner to the history as a new event, lets the newest event attend and so accumulate what weight the blocks draw, and
cuts histories that outgrow their budget.  The events' keys are item embeddings, their values the embeddings again: a
stand-in for the trained projections of a ranking model.  Prints one JSON line.
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
    handed out and taken back, and copied to the device for a call; the blocks' accumulated weights stay there."""

    def __init__(self, n_users: int, n_pages: int, n_heads: int, d: int, max_blocks: int):
        self.cache = st.KvCache.empty(n_pages, n_heads, d)
        self.max_blocks = max_blocks
        self.tables = np.full((n_users, max_blocks), -1, np.int32)
        self.lengths = np.zeros(n_users, np.int32)
        self.mass = torch.zeros((n_users, n_heads, max_blocks), dtype=torch.float32, device="cuda")
        self.free = list(range(n_pages - 1, -1, -1))

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
        taken = int((need - have).sum())
        if taken > len(self.free):
            raise ValueError(f"{taken} pages are needed, {len(self.free)} are free: evict first")
        pages = iter(self.free[len(self.free) - taken:][::-1])
        for row, a, b in zip(tables, have, need):
            for block in range(a, b):
                row[block] = next(pages)
        lengths = (lengths + counts).astype(np.int32)
        st.st_kv_append(self.cache, self._view(tables, lengths, counts), k, v)
        self.tables[users], self.lengths[users] = tables, lengths
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
        for i, n in enumerate(count):
            self.free.extend(pages[i, :n].tolist())
        return int(count.sum())


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--items", type=int, default=200_000)
    ap.add_argument("--users", type=int, default=64)
    ap.add_argument("--events", type=int, default=3000)
    ap.add_argument("--candidates", type=int, default=100)
    ap.add_argument("--select", type=int, default=8, help="blocks each candidate reads in every other step (0: always all)")
    ap.add_argument("--budget", type=int, default=40, help="blocks a history may hold")
    ap.add_argument("--steps", type=int, default=8)
    args = ap.parse_args()
    from paper_2511_14881_amd import synth

    if not torch.cuda.is_available():
        print("history needs a GPU", file=sys.stderr)
        sys.exit(2)
    cfg = synth.scaled(synth.CONFIGS["mid"], args.items, batch=args.users, top_k=args.candidates)
    w = synth.make_workload(cfg, device="cuda")
    bloom = st.st_bloom_build(w.feat_offsets, w.feat_ids, cfg.n_items, cfg.m_bits, cfg.k_hashes)
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
