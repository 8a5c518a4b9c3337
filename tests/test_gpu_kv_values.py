"""Attention over cached histories whose values are as large or as small as bf16 holds, against the definition in 64 bits (kv_wide): outputs are
averages of values, so they are finite wherever the values are.  The bound is test_gpu_kv_scales'."""
import numpy as np
import pytest
import torch

from paper_2511_14881_amd import binding as st
from tests import kv_reference as R
from tests import kv_wide as W
from tests.test_gpu_kv import queries, say

pytestmark = pytest.mark.gpu

# value scales of the blocks, in turn (127 of the largest is 3.3e38, just below the largest finite number)
ORDERS = {
    "largest": [2.6e36],
    "large": [2e36, 1e33, 2.6e36, 1e34, 1e35],
    "large late": [0.02, 0.5, 3.0, 1e-3, 0.01, 0.04, 1.0, 2.0, 0.3, 2.5e36, 0.02, 1e20, 7.0],
    "smallest": [1e-38],
    "small": [2e-38, 3e-37, 1e-38, 4e-36],
}


@pytest.mark.parametrize("lens,n_q", [([64 * 40, 64 * 40 - 3, 700], 1), ([20000], 2), ([64 * 40, 64 * 40 - 3, 700], 110), ([9000], 200)])  # whole and split
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("order", list(ORDERS))
def test_values_of_extreme_size(order, d, lens, n_q):
    say(f"[kv] values {order} d={d} lens={lens} n_q={n_q}")
    rng = np.random.default_rng(d + n_q)
    host = R.Host(rng, lens, 2, d)
    for s, n in enumerate(lens):
        for b in range(-(-n // 64)):
            host.vs[host.tables[s, b]] = ORDERS[order][(b + s) % len(ORDERS[order])]
    n_tok = n_q * len(lens)
    q = queries(rng, n_tok, 6, d, "bf16")
    out = st.st_kv_attend(host.cache(st), host.batch(st, n_tok, max_len=max(lens)), q.cuda(), causal=False)
    want, _, _, reach, value = W.attend(host, q, d ** -0.5, False)
    W.check(out, want, W.error(host, want, reach, value, "bf16"))
    blocks = st.st_kv_select(host.cache(st), host.batch(st, n_tok, max_len=max(lens)), q[:, :6].cuda(), 20, causal=False)
    out = st.st_kv_attend(host.cache(st), host.batch(st, n_tok, max_len=max(lens)), q.cuda(), causal=False, blocks=blocks)
    want, _, _, reach, value = W.attend(host, q, d ** -0.5, False, blocks=blocks.cpu().numpy())
    W.check(out, want, W.error(host, want, reach, value, "bf16"))


@pytest.mark.parametrize("scale", [2.6e36, 1e-38])
@pytest.mark.parametrize("d,group,n_q", [(64, 4, 1), (128, 4, 4), (64, 1, 130), (256, 1, 100)])
def test_long_histories_of_extreme_values(d, group, n_q, scale):
    """65536 tokens of one size to a workgroup that walks them all, weights near one another."""
    rng = np.random.default_rng(51)
    heads, n, n_seq = 4, 65536, {1: 256, 4: 128, 130: 64, 100: 64}[n_q]
    host = R.Host(rng, [n], heads, d)
    host.vs[:] = np.float32(scale)
    host.v[:] = np.abs(host.v.astype(np.int16)).clip(1, 127)
    W.shared(host, [n] * n_seq)
    q = queries(rng, n_q, heads * group, d, "bf16", 0.2)
    out = st.st_kv_attend(host.cache(st), host.batch(st, n_q * n_seq), q.repeat(n_seq, 1, 1).cuda(), causal=False)
    want, _, _, reach, value = W.attend(W.part(host, [0]), q, d ** -0.5, False)
    for s in (0, n_seq - 1):
        W.check(out[s * n_q:(s + 1) * n_q], want, W.error(host, want, reach, value, "bf16"))
