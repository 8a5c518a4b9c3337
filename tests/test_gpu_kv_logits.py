"""Attention over cached histories with logits and queries of any finite size, against the definition in 64 bits (kv_wide)."""
import numpy as np
import pytest
import torch

from paper_2511_14881_amd import binding as st
from tests import kv_reference as R
from tests import kv_wide as W
from tests.test_gpu_kv import queries, say

pytestmark = pytest.mark.gpu
SHAPES = [(64, 4, 1), (128, 4, 1), (256, 2, 3), (64, 3, 120), (96, 5, 60), (128, 2, 200), (256, 3, 100)]  # d, group, n_q: few rows, many rows


@pytest.mark.parametrize("size", [1e3, 1e5, 3e6, 1e8, 1e11, 1e20])
@pytest.mark.parametrize("d,group,n_q", SHAPES)
def test_large_logits_choose_one_token(d, group, n_q, size):
    """Rows whose largest logit is further above the second than what rounding in fp32 can be off by, and 40 nats: the output is that token's value."""
    say(f"[kv] logits of size {size} d={d} group={group} n_q={n_q}")
    rng = np.random.default_rng(41)
    host = R.Host(rng, [1500, 1100, 333], 2, d)
    n_tok = 3 * n_q
    q = queries(rng, n_tok, 2 * group, d, "bf16", size)
    lse = torch.zeros((n_tok, 2 * group), device="cuda")
    out = st.st_kv_attend(host.cache(st), host.batch(st, n_tok, max_len=1500), q.cuda(), causal=False, lse=lse)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    got, q64, rows = out.float().cpu().numpy(), R.to_float(q), 0
    for tok in range(n_tok):
        for h in range(2):
            k, v = host.rows(tok // n_q, h)
            for g in range(h * group, (h + 1) * group):
                x = k @ q64[tok, g] * d ** -0.5
                order = np.argsort(x)[::-1]
                off = 2 * (d + 8) * 2.0 ** -24 * (np.abs(k) @ np.abs(q64[tok, g])).max() * d ** -0.5
                if x[order[0]] - x[order[1]] > off + 40:
                    rows += 1
                    value = v[order[0]]
                    others = len(x) * np.exp(-40.0) * np.abs(v).max()
                    assert np.all(np.abs(got[tok, g] - value) <= 2.0 ** -8 * np.abs(value) + others), (tok, g)
                    assert abs(lse[tok, g].item() - x[order[0]]) <= off + 2.0 ** -20 * abs(x[order[0]])
    assert rows > n_tok * 2 * group / 2


@pytest.mark.parametrize("d,group,n_q", SHAPES)
def test_equal_large_logits_share_the_weight(d, group, n_q):
    """All keys of a history are one key: the weights are equal however large the logits."""
    rng = np.random.default_rng(42)
    host = R.Host(rng, [1000, 130], 2, d)
    host.k[:] = host.k[host.tables[0, 0], :1, :1]
    host.ks[:] = np.float32(0.0371)
    for size in (1e3, 1e6, 1e9, 1e15):
        q = queries(rng, 2 * n_q, 2 * group, d, "bf16", size)
        out = st.st_kv_attend(host.cache(st), host.batch(st, 2 * n_q, max_len=1000), q.cuda(), causal=False)
        want = np.zeros(out.shape)
        value = np.zeros(out.shape[:2])
        for s in range(2):
            for h in range(2):
                want[s * n_q:(s + 1) * n_q, h * group:(h + 1) * group] = host.rows(s, h)[1].mean(0)
                value[s * n_q:(s + 1) * n_q, h * group:(h + 1) * group] = 127.0 * host.vs[host.tables[s, : -(-host.lens[s] // 64)], h].max()
        W.check(out, want, W.error(host, want, np.zeros(value.shape), value, "bf16"))


@pytest.mark.parametrize("d,group,n_q", SHAPES)
def test_queries_up_to_the_largest_number(d, group, n_q):
    """bf16 queries from 2^117 up to its largest finite number, with keys that bring the logits back to ordinary size."""
    rng = np.random.default_rng(43)
    host = R.Host(rng, [900, 300], 2, d)
    host.ks[:] = rng.uniform(2e-38, 4e-38, host.ks.shape)
    for size in (2e35, 4e36, 6e37):
        q = queries(rng, 2 * n_q, 2 * group, d, "bf16", size)
        q[0, 0, 0] = torch.finfo(torch.bfloat16).max
        assert torch.isfinite(q).all()
        scale = 1.0 / (size * 3e-38 * 40 * d ** 0.5)
        out = st.st_kv_attend(host.cache(st), host.batch(st, 2 * n_q, max_len=900), q.cuda(), scale=scale, causal=False)
        want, _, _, reach, value = W.attend(host, q, scale, False)
        W.check(out, want, W.error(host, want, reach, value, "bf16"))
