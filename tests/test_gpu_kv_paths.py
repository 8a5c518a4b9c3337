"""Every path through the kernels on cached histories, at sizes that reach it: walks of many blocks and several rounds of them, each kernel that
chooses, joins and sums.  Sequences share the pages of one long history, so that large calls need little memory; some of
them are compared with the definition in 64 bits (kv_wide, kv_reference), the bounds are test_gpu_kv's."""
import numpy as np
import pytest
import torch

from paper_2511_14881_amd import binding as st
from tests import kv_reference as R
from tests import kv_wide as W
from tests.test_gpu_kv import TYPES, check_out, cuda_mask, queries, say

pytestmark = pytest.mark.gpu


def ragged(n_seq, top):
    """Lengths from top down to a quarter of it, in no order, one of them 1."""
    lens = [top - (i * 37 % n_seq) * 3 * top // (4 * n_seq) for i in range(n_seq)]
    lens[n_seq // 2] = 1
    return lens


def rows_of(seqs, n_q):
    return np.concatenate([np.arange(s * n_q, (s + 1) * n_q) for s in seqs])


def bits(rng, n_tok, words, kind):
    """None, or masks: "rounds" leaves whole runs of 64 blocks empty for all rows, others for some."""
    if kind is None:
        return None
    m = rng.integers(0, 1 << 64, (n_tok, words), dtype=np.uint64)
    m[rng.random((n_tok, words)) < 0.5] = 0
    m[rng.random(n_tok) < 0.1] = 0
    if kind == "rounds":
        m[:, 64:128] = 0
        m[:, 5:9] = 0
        m[: n_tok // 2, 130:] = 0
    return m


ATTEND = {
    # dtype, d, heads, group, lens, n_q, causal, mask, compared sequences
    # tiles of 16 rows, a wavefront each: from 2048 tiles on
    "one wavefront": ("bf16", 128, 8, 4, ragged(64, 64 * 70 + 9), 16, True, None, [0, 32, 63]),
    "one wavefront, mask": ("f16", 64, 8, 8, ragged(44, 9000), 12, False, "rounds", [0, 22]),
    "one wavefront, all rows in a tile": ("f16", 96, 4, 3, ragged(520, 700), 1, True, "any", [0, 1, 260, 519]),
    "one wavefront, d = 256": ("bf16", 256, 4, 5, ragged(104, 64 * 66), 16, True, None, [0, 52]),
    # four wavefronts: more than 256 blocks to a split
    "long splits": ("bf16", 128, 8, 4, ragged(64, 64 * 300 + 1), 1, True, None, [0, 1, 32]),
    "long splits, mask": ("f16", 64, 8, 2, ragged(128, 64 * 280), 1, True, "rounds", [0, 64]),
    "long splits, d = 96": ("bf16", 96, 8, 1, ragged(100, 64 * 270 + 5), 2, False, None, [0, 99]),
    "long splits, d = 256": ("f16", 256, 8, 2, ragged(64, 64 * 262 + 63), 1, True, "any", [0, 63]),
    # the thresholds between few and many rows where there is much to do
    "few rows, d = 64": ("bf16", 64, 4, 4, ragged(8, 8000), 32, True, None, [0, 4]),
    "few rows, d = 96": ("f16", 96, 4, 4, ragged(8, 8000), 32, True, "any", [0, 4]),
    "few rows, d = 256": ("bf16", 256, 4, 3, ragged(8, 8000), 32, True, None, [0, 4]),
    # many rows: walks of hundreds of blocks
    "many rows": ("bf16", 128, 8, 2, ragged(32, 64 * 150 + 3), 80, False, None, [0, 16]),
    "many rows, causal": ("f16", 64, 8, 1, ragged(32, 64 * 140), 190, True, None, [0, 16]),
    "many rows, mask": ("bf16", 96, 8, 3, ragged(32, 64 * 200 + 17), 50, True, "rounds", [0, 16]),
    "many rows, mask, d = 128": ("f16", 128, 8, 1, ragged(32, 64 * 140), 201, True, "rounds", [0, 16]),
    "many rows, d = 256": ("bf16", 256, 8, 2, ragged(32, 64 * 135), 60, True, None, [0, 16]),
    "many rows, mask, d = 256": ("f16", 256, 8, 1, ragged(32, 64 * 190), 101, False, "rounds", [0, 16]),
    "many rows, few blocks to a workgroup": ("bf16", 128, 2, 4, ragged(3, 5000), 90, True, "any", [0, 2]),
    # joins of 16 splits and more, of few and of many rows
    "join, d = 64": ("bf16", 64, 2, 4, [20011], 1, True, None, [0]),
    "join, d = 96": ("bf16", 96, 1, 2, [20011], 3, True, "any", [0]),
    "join, d = 256": ("f16", 256, 2, 2, [20011, 300], 2, True, "any", [0, 1]),
    "join, many rows, d = 64": ("f16", 64, 1, 2, [30000], 170, True, None, [0]),
    "join, many rows, d = 256": ("bf16", 256, 1, 3, [30000], 90, True, "any", [0]),
}


@pytest.mark.parametrize("extra", [False, True])  # lse and accumulated weights too
@pytest.mark.parametrize("name", list(ATTEND))
def test_attention_on_every_path(name, extra):
    dtype, d, heads, group, lens, n_q, causal, kind, seqs = ATTEND[name]
    say(f"[kv] path {name}, extra={extra}")
    rng = np.random.default_rng(500 + list(ATTEND).index(name))
    host = W.shared(R.Host(rng, [max(lens)], heads, d), lens)
    n_tok = n_q * len(lens)
    q = queries(rng, n_tok, heads * group, d, dtype)
    mask = bits(rng, n_tok, host.max_blocks, kind)
    cache, batch = host.cache(st), host.batch(st, n_tok, max_len=max(lens))
    args = {}
    if extra:
        args = {"lse": torch.full((n_tok, heads * group), 7.0, device="cuda"), "decay": 0.75,
                "mass_out": torch.full((len(lens), heads, host.max_blocks), 7.0, device="cuda")}
        mass = rng.uniform(0, 3, tuple(args["mass_out"].shape)).astype(np.float32)
        args["mass"] = torch.from_numpy(mass).cuda()
    out = torch.full((n_tok, heads * group, d), 7.0, dtype=TYPES[dtype], device="cuda")
    st.st_kv_attend(cache, batch, q.cuda(), causal=causal, mask=cuda_mask(mask), out=out, **args)
    torch.cuda.synchronize()
    at = rows_of(seqs, n_q)
    some = W.part(host, seqs)
    want, want_lse, want_mass, reach, _ = W.attend(some, q[at], d ** -0.5, causal, mask=None if mask is None else mask[at],
                                                   mass=mass[seqs] if extra else None, decay=0.75)
    check_out(out[torch.from_numpy(at).cuda()], want, reach, some, dtype)
    assert torch.isfinite(out).all()
    if extra:
        got = args["lse"].cpu().numpy()[at].astype(np.float64)
        fin = np.isfinite(want_lse)
        assert np.array_equal(np.isneginf(got), ~fin)
        assert np.all(np.abs(got - np.where(fin, want_lse, 0))[fin] <= W.lse_error(some, want_lse, reach)[fin])
        rows = n_q * group
        rel = (4 * (d + 8) * reach.max(initial=0) + max(lens) / 8 + 128 + rows) * 2.0 ** -23
        assert np.all(np.abs(args["mass_out"].cpu().numpy()[seqs] - want_mass) <= rel * rows + 2.0 ** -22 * want_mass + 1e-30)
    again = out.clone()
    st.st_kv_attend(cache, batch, q.cuda(), causal=causal, mask=cuda_mask(mask), out=out, **args)
    assert torch.equal(again, out)


SELECT = {
    # dtype, d, heads, group, lens, n_q, causal, mask, n_sel, sink, recent, compared sequences
    # several tokens: keys in memory, then a wavefront of 4, 8 or 16 keys a lane, or a workgroup, chooses
    "200 blocks": ("bf16", 64, 2, 2, ragged(3, 64 * 200), 5, True, None, 9, 1, 2, [0, 1, 2]),
    "300 blocks": ("f16", 128, 2, 3, ragged(3, 64 * 300 - 7), 17, True, "rounds", 20, 0, 3, [0, 1, 2]),
    "700 blocks": ("bf16", 96, 1, 4, ragged(3, 64 * 700), 3, False, "any", 33, 2, 0, [0, 1, 2]),
    "1500 blocks": ("f16", 256, 2, 1, ragged(2, 64 * 1500 + 11), 3, True, "rounds", 70, 3, 3, [0, 1]),
    "3000 blocks": ("bf16", 64, 1, 2, [64 * 3000], 2, True, None, 1500, 1, 1, [0]),
    # a workgroup scores several rounds of 256 blocks
    "rounds": ("bf16", 64, 8, 1, ragged(64, 64 * 700), 3, True, "any", 12, 1, 1, [0, 32]),
    "chunks and rounds": ("f16", 128, 4, 2, ragged(40, 64 * 900), 4, True, None, 25, 0, 0, [0, 20]),
    "rounds, 1500 blocks": ("bf16", 96, 8, 2, ragged(64, 64 * 1500), 2, False, None, 64, 2, 2, [0, 32]),
    # one token a sequence: one kernel, second round of 512 blocks; more than 1024 blocks with and without as many pairs as compute units
    "a token, 700 blocks": ("f16", 64, 2, 4, ragged(3, 64 * 700 + 1), 1, True, "any", 18, 1, 2, [0, 1, 2]),
    "a token, 1024 blocks": ("bf16", 128, 2, 4, ragged(3, 64 * 1024), 1, True, None, 64, 1, 2, [0, 1, 2]),
    "a token, d = 256": ("bf16", 256, 2, 4, ragged(3, 64 * 520 + 1), 1, True, "any", 12, 1, 1, [0, 1, 2]),
    "a token, 1100 blocks": ("bf16", 64, 4, 2, ragged(64, 64 * 1100 - 5), 1, True, "rounds", 30, 1, 2, [0, 1, 32]),
    "a token, 5000 blocks": ("f16", 96, 4, 1, ragged(64, 64 * 5000), 1, False, None, 300, 0, 4, [0, 32]),
    "a token, 5000 blocks, one sequence": ("f16", 256, 1, 2, [64 * 5000 - 1], 1, True, "any", 100, 5, 4, [0]),
    "a token, 16384 blocks": ("bf16", 64, 1, 1, [64 * 16384], 1, True, None, 2000, 1, 1, [0]),
    # attention over what was selected: a wavefront to a tile, more than 64 selected blocks; four wavefronts, more than 256
    "lookups": ("f16", 128, 4, 1, ragged(8, 20000), 70, False, "any", 8, 0, 1, [0, 4]),
    "lookups, 70 blocks": ("bf16", 64, 4, 20, ragged(8, 9000), 35, True, None, 70, 1, 1, [0, 4]),
    "lookups, d = 96": ("bf16", 96, 8, 2, ragged(8, 9000), 40, True, "rounds", 66, 1, 1, [0, 4]),
    "lookups, d = 256": ("f16", 256, 4, 2, ragged(8, 9000), 70, False, None, 6, 1, 1, [0, 4]),
    "270 of 300 blocks": ("bf16", 128, 8, 2, ragged(32, 64 * 300), 2, True, None, 270, 1, 1, [0, 16]),
}


@pytest.mark.parametrize("name", list(SELECT))
def test_selection_and_attention_over_it_on_every_path(name):
    dtype, d, heads, group, lens, n_q, causal, kind, n_sel, sink, recent, seqs = SELECT[name]
    say(f"[kv] select path {name}")
    rng = np.random.default_rng(700 + list(SELECT).index(name))
    host = W.shared(R.Host(rng, [max(lens)], heads, d), lens)
    host.bounds[::3] = host.bounds[0]  # scores that are equal, and others that are close
    host.ks[::3] = np.where(np.isnan(host.ks[::3]), np.nan, np.float32(0.03))
    n_tok = n_q * len(lens)
    q = queries(rng, n_tok, heads * group, d, dtype)
    mask = bits(rng, n_tok, host.max_blocks, kind)
    cache, batch = host.cache(st), host.batch(st, n_tok, max_len=max(lens))
    blocks = st.st_kv_select(cache, batch, q.cuda(), n_sel, causal=causal, mask=cuda_mask(mask), sink=sink, recent=recent)
    torch.cuda.synchronize()
    at = rows_of(seqs, n_q)
    some, some_mask = W.part(host, seqs), None if mask is None else mask[at]
    want = R.select(some, q[at], n_sel, causal, sink, recent, mask=some_mask)
    assert np.array_equal(blocks.cpu().numpy()[at], want)
    mass_out = torch.full((len(lens), heads, host.max_blocks), 7.0, device="cuda")
    out = st.st_kv_attend(cache, batch, q.cuda(), causal=causal, mask=cuda_mask(mask), blocks=blocks, mass_out=mass_out)
    again = st.st_kv_attend(cache, batch, q.cuda(), causal=causal, mask=cuda_mask(mask), blocks=blocks)
    torch.cuda.synchronize()
    assert torch.equal(out, again)
    ref, _, ref_mass, reach, _ = W.attend(some, q[at], d ** -0.5, causal, mask=some_mask, blocks=want)
    check_out(out[torch.from_numpy(at).cuda()], ref, reach, some, dtype)
    rows = n_q * group
    rel = (4 * (d + 8) * reach.max(initial=0) + max(lens) / 8 + 128 + rows) * 2.0 ** -23
    assert np.all(np.abs(mass_out.cpu().numpy()[seqs] - ref_mass) <= rel * rows + 2.0 ** -22 * ref_mass + 1e-30)


@pytest.mark.parametrize("d,group", [(64, 1), (96, 4), (128, 2), (256, 3)])
def test_different_numbers_of_tokens_in_one_call(d, group):
    """A prompt's chunk, candidates, single tokens and none beside one another; max_tok as it is, and n_tok in its place."""
    rng = np.random.default_rng(92)
    counts, lens = [301, 1, 0, 20, 1, 77, 2], [2000, 9000, 500, 640, 1, 4100, 0]
    offsets = np.concatenate([[0], np.cumsum(counts)]).tolist()
    host = R.Host(rng, lens, 2, d)
    n_tok = offsets[-1]
    q = queries(rng, n_tok, 2 * group, d, "bf16")
    mass = rng.uniform(0, 3, (len(lens), 2, host.max_blocks)).astype(np.float32)
    cache, want, results = host.cache(st), W.attend(host, q, d ** -0.5, True, offsets=offsets, mass=mass, decay=0.5), []
    chosen = R.select(host, q, 5, True, 1, 1, offsets)
    for kw in ({"max_tok": 301}, {}):
        batch = host.batch(st, n_tok, offsets, **kw)
        mass_out = torch.full(mass.shape, 7.0, device="cuda")
        out = st.st_kv_attend(cache, batch, q.cuda(), mass=torch.from_numpy(mass).cuda(), decay=0.5, mass_out=mass_out)
        check_out(out, want[0], want[3], host, "bf16")
        rows = 301 * group
        rel = (4 * (d + 8) * want[3].max() + 9000 / 8 + 128 + rows) * 2.0 ** -23
        assert np.all(np.abs(mass_out.cpu().numpy() - want[2]) <= rel * rows + 2.0 ** -22 * want[2] + 1e-30)
        blocks = st.st_kv_select(cache, batch, q.cuda(), 5, sink=1, recent=1)
        assert np.array_equal(blocks.cpu().numpy(), chosen)
        results.append(st.st_kv_attend(cache, batch, q.cuda(), blocks=blocks))
    ref, _, _, reach, _ = W.attend(host, q, d ** -0.5, True, offsets=offsets, blocks=chosen)
    for out in results:
        check_out(out, ref, reach, host, "bf16")


@pytest.mark.parametrize("scale", [-0.1, 0.0, 1e-30])
@pytest.mark.parametrize("d,group,n_q", [(64, 4, 1), (128, 2, 200), (256, 3, 100)])
def test_scales_of_either_sign_and_none(scale, d, group, n_q):
    rng = np.random.default_rng(90)
    host = R.Host(rng, [1500, 333], 2, d)
    q = queries(rng, 2 * n_q, 2 * group, d, "bf16")
    lse = torch.zeros((2 * n_q, 2 * group), device="cuda")
    out = st.st_kv_attend(host.cache(st), host.batch(st, 2 * n_q, max_len=1500), q.cuda(), scale=scale, lse=lse)
    want, want_lse, _, reach, _ = W.attend(host, q, scale, True)
    check_out(out, want, np.maximum(reach, 1e-30), host, "bf16")
    assert np.all(np.abs(lse.cpu().numpy() - want_lse) <= W.lse_error(host, want_lse, reach))


@pytest.mark.parametrize("n_q", [1, 60, 300])
def test_weights_without_earlier_ones(n_q):
    rng = np.random.default_rng(91)
    host = R.Host(rng, [900, 64, 2000], 2, 64)
    q = queries(rng, 3 * n_q, 4, 64, "f16")
    out = torch.full((3, 2, host.max_blocks), 7.0, device="cuda")
    st.st_kv_attend(host.cache(st), host.batch(st, 3 * n_q, max_len=2000), q.cuda(), causal=False, mass_out=out)
    _, _, want, reach, _ = W.attend(host, q, 64 ** -0.5, False)
    rows = 2 * n_q
    rel = (4 * 72 * reach.max() + 2000 / 8 + 128 + rows) * 2.0 ** -23
    assert np.all(np.abs(out.cpu().numpy() - want) <= rel * rows + 2.0 ** -22 * want + 1e-30)
