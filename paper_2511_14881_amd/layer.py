"""A layer of the attention models on either side of the search, around users' cached histories: rows are normalised into int8
(``st_norm_rows``), projected to queries, keys and values with each tenant's adapter (``st_project``), given their positions
(``st_rotate``), appended to the histories and attended with (``HistoryStore``), and projected back.  The last norm's int8 rows
are the search's queries."""
from __future__ import annotations

import torch

from paper_2511_14881_amd import binding as st
from paper_2511_14881_amd.history import HistoryStore


class Projection:
    """Weights w [n, k] held as int8 rows with a scale each, and a low-rank adapter for each tenant: a [tenants, rank, k],
    b [tenants, n, rank] of the outputs' type, alpha fp32 [tenants]."""

    def __init__(self, w: torch.Tensor, a: torch.Tensor | None = None, b: torch.Tensor | None = None, alpha: torch.Tensor | None = None):
        rows = st.st_norm_rows(w, normalise=False)
        self.w, self.scale = rows.q, rows.scale
        self.adapters = None if a is None else st.Adapters(a, b, alpha)

    def __call__(self, rows: st.NormRows, tenants: torch.Tensor | None, dtype) -> torch.Tensor:
        """The rows' projection; tenants int32 [n_rows] (-1: no adapter), or None for none at all."""
        adapters = self.adapters if tenants is not None else None
        return st.st_project(rows.q, rows.scale, self.w, self.scale, adapters, tenants if adapters is not None else None, dtype=dtype)


class HistoryLayer:
    """heads query heads share the store's kv_heads heads of d values.  norm [width], w_qkv [(heads + 2 kv_heads) d, width] and w_out
    [width out, heads d] are of the layer's type (bf16 or fp16), each with adapters (a, b, alpha) if given; sections and freqs: the
    axes of the positions (``st_rotate``)."""

    def __init__(self, heads: int, kv_heads: int, d: int, norm, w_qkv, w_out, sections, freqs, qkv_adapters=(), out_adapters=(), eps: float = 1e-6):
        if heads < 1 or kv_heads < 1 or heads % kv_heads or w_qkv.shape[0] != (heads + 2 * kv_heads) * d or w_out.shape[1] != heads * d:
            raise ValueError("w_qkv must be [(heads + 2 kv_heads) d, width] and w_out [width, heads d], heads a multiple of kv_heads")
        self.heads, self.kv_heads, self.d, self.eps = heads, kv_heads, d, eps
        self.norm, self.sections, self.freqs = norm, tuple(int(s) for s in sections), freqs
        self.qkv, self.out = Projection(w_qkv, *qkv_adapters), Projection(w_out, *out_adapters)

    def project(self, x, positions, tenants=None, residual=None):
        """Queries, keys and values of the rows x [n, width], rotated: views of one tensor; and the rows' sum with the residual."""
        rows = st.st_norm_rows(x, self.norm, residual, eps=self.eps)
        qkv = self.qkv(rows, tenants, x.dtype).view(x.shape[0], self.heads + 2 * self.kv_heads, self.d)
        q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=1)
        st.st_rotate(q, k, positions, self.freqs, self.sections, out=(q, k))
        return q, k, v, x if residual is None else rows.total

    def take_in(self, store: HistoryStore, users, x, positions, counts=None, tenants=None) -> None:
        """Events x [sum of counts, width] behind the users' histories, without attending."""
        _, k, v, _ = self.project(x, positions, tenants)
        store.append(users, k, v, counts)

    def __call__(self, store: HistoryStore, users, x, positions, counts=None, tenants=None, residual=None, append: bool = True, **attend):
        """The rows' outputs and their sum with the residual.  append: the rows are events that join the histories and attend to what comes
        before them, and to themselves; otherwise they (candidates) attend to the histories as they are.  attend: of
        ``HistoryStore.attend`` (n_sel, track, decay, ...)."""
        q, k, v, total = self.project(x, positions, tenants, residual)
        if append:
            store.append(users, k, v, counts)
        counts = [1] * len(users) if counts is None else counts
        seen = store.attend(users, q, counts, causal=append, **attend)
        rows = st.st_norm_rows(seen.view(x.shape[0], self.heads * self.d), normalise=False)
        return self.out(rows, tenants, x.dtype), total
