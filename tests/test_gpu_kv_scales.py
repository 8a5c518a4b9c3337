"""Attention over cached histories whose blocks differ in the scale of their values, against the definition in 64 bits (kv_wide).  The bound is
test_gpu_kv's, with V the largest value of the blocks that the row itself sees."""
import numpy as np
import pytest
import torch

from paper_2511_14881_amd import binding as st
from tests import kv_reference as R
from tests import kv_wide as W
from tests.test_gpu_kv import cuda_mask, queries, say

pytestmark = pytest.mark.gpu

# value scales of the blocks, in turn: falling, rising and both ways, by little and by much
ORDERS = {
    "one tiny": [0.02, 0.02, 1e-36, 0.02],
    "all sizes": [0.02, 1e-36, 0.02, 1.0, 3e-3, 0.0, 1e-30, 7.0, 1e-10, 0.3, 1e-3, 1e-38],
    "falling": [1.0, 0.24, 0.06, 0.015, 1e-3, 2e-5, 1e-9, 1e-18, 1e-30],
    "rising": [0.0, 1e-37, 1e-30, 1e-12, 1e-5, 1e-3, 0.01, 0.019, 0.1, 2.0],
    "near": [0.02, 0.012, 0.0101, 0.0051, 0.0049, 0.0201, 0.037, 0.039, 0.0097],
}


@pytest.mark.parametrize("n_q", [1, 110])  # few rows, many rows
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("order", list(ORDERS))
def test_value_scales_of_all_sizes(order, d, n_q):
    say(f"[kv] value scales {order} d={d} n_q={n_q}")
    rng = np.random.default_rng(d + n_q)
    heads, group, lens = 2, 3, [64 * 48 + 5, 64 * 48, 700, 64 * 30, 2000, 64 * 47, 64 * 40, 3000]
    host = R.Host(rng, lens, heads, d)
    for s, n in enumerate(lens):
        for b in range(-(-n // 64)):
            host.vs[host.tables[s, b]] = ORDERS[order][(b + s) % len(ORDERS[order])]
    n_tok = n_q * len(lens)
    q = queries(rng, n_tok, heads * group, d, "bf16")
    # a third of the tokens sees one block in seven, or nothing
    mask = np.full((n_tok, host.max_blocks), ~np.uint64(0))
    for tok in range(0, n_tok, 3):
        mask[tok, (np.arange(host.max_blocks) + tok) % 7 != 0] = 0
    mask[n_tok // 2] = 0
    lse = torch.zeros((n_tok, heads * group), device="cuda")
    out = st.st_kv_attend(host.cache(st), host.batch(st, n_tok, max_len=max(lens)), q.cuda(), causal=False, mask=cuda_mask(mask), lse=lse)
    plain = st.st_kv_attend(host.cache(st), host.batch(st, n_tok, max_len=max(lens)), q.cuda(), causal=False)
    want, want_lse, _, reach, value = W.attend(host, q, d ** -0.5, False, mask=mask)
    W.check(out, want, W.error(host, want, reach, value, "bf16"))
    fin = np.isfinite(want_lse)
    assert np.all(np.abs(lse.cpu().numpy() - np.where(fin, want_lse, 0))[fin] <= W.lse_error(host, want_lse, reach)[fin])
    want, _, _, reach, value = W.attend(host, q, d ** -0.5, False)
    W.check(plain, want, W.error(host, want, reach, value, "bf16"))


@pytest.mark.parametrize("ratio", [250.0, 100.0, 3.9])
def test_many_light_tokens_in_blocks_of_small_scale_count_in_full(ratio):
    """One token far above 65535 others whose values have a smaller scale: the others' weights are a few units of a 16-bit float's last place
    where the scales' ratio is part of them, and make up a part of the sum all the same.  One workgroup walks all blocks."""
    rng = np.random.default_rng(31)
    heads, d, n, n_seq, n_q = 8, 64, 65536, 32, 130
    host = R.Host(rng, [n], heads, d)
    host.k[:] = 0
    host.ks[:] = np.float32(0.01)
    host.vs[:] = np.float32(1.0 / ratio)
    first = host.tables[0, 0]
    host.k[first, :, 5] = 100
    host.v[first, :, 5] = 127
    host.vs[first] = 1.0
    # the first token lies 14 to 17 nats above the others, which weigh 0.5 to 0.03 of it in all
    q = torch.from_numpy(np.broadcast_to(np.linspace(14.0, 17.0, n_q)[:, None, None] / 8.0, (n_q, heads, d)).astype(np.float32)).to(torch.float16)
    W.shared(host, [n] * n_seq)
    every = q.repeat(n_seq, 1, 1)
    out = st.st_kv_attend(host.cache(st), host.batch(st, n_q * n_seq), every.cuda(), causal=False)
    assert all(torch.equal(out[:n_q], out[i * n_q:(i + 1) * n_q]) for i in range(1, n_seq))
    want, _, _, reach, value = W.attend(W.part(host, [0]), q, d ** -0.5, False)
    W.check(out[:n_q], want, W.error(host, want, reach, value, "f16"))
