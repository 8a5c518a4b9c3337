"""The operators on cached histories through the C ABI against the plain implementation in 64 bits (kv_reference).

Whole numbers (selected blocks, what an append writes, what an eviction keeps) are compared bit for bit.  For outputs of attention
the bound is derived, element by element, for a row with S = max over its tokens of sum |q_c k_c| * scale and V = max |v|:
  - the output's rounding to 16 bits: 2^-9 |out| (bf16) or 2^-12 |out| + 2^-25 (fp16), taken twice
  - the weights' rounding to 11 significant bits: 2^-12 V
  - fp32 logits: d + 8 roundings of partial sums at most S, so a weight is off by a factor 2 (d + 8) S 2^-24
  - fp32 sums over T tokens of weights and products, at most (T / 16 + 64) roundings each: (T / 16 + 64) 2^-23 V
"""
import numpy as np
import pytest
import torch

from paper_2511_14881_amd import binding as st
from tests import kv_reference as R

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def say(*a):
    print(*a, flush=True)


def queries(rng, n_tok, n_qh, d, dtype, size=1.0):
    return torch.from_numpy(rng.normal(0, size, (n_tok, n_qh, d)).astype(np.float32)).to(TYPES[dtype])


def masks(rng, n_tok, words, kind):
    if kind is None:
        return None
    m = rng.integers(0, 1 << 64, (n_tok, words), dtype=np.uint64)
    if kind == "sparse":
        for _ in range(4):
            m &= rng.integers(0, 1 << 64, (n_tok, words), dtype=np.uint64)
    m[rng.random((n_tok, words)) < 0.4] = 0
    m[rng.random(n_tok) < 0.25] = 0  # rows that see nothing
    m[-1, :] = 0
    return m


def cuda_mask(m):
    return None if m is None else torch.from_numpy(m.view(np.int64)).cuda()


def check_out(got, want, reach, host, dtype):
    got = got.float().cpu().numpy().astype(np.float64)
    vmax = 128.0 * np.nanmax(host.vs) if np.isfinite(host.vs).any() else 0.0
    T = max(host.lens)
    rel = (2 * (host.d + 8) * reach * 2.0 ** -24 + 2.0 ** -12 + (T / 16 + 64) * 2.0 ** -23)[..., None]
    half = 2.0 ** -8 * np.abs(want) if dtype == "bf16" else 2.0 ** -11 * np.abs(want) + 2.0 ** -24
    assert np.isfinite(got).all()
    over = np.abs(got - want) - (rel * vmax + half)
    assert over.max(initial=-1.0) <= 0, f"off by {np.abs(got - want).max()} at {np.unravel_index(over.argmax(), over.shape)}"
    assert np.all(got[reach == 0] == 0)


CASES = [
    # dtype, d, heads, group, lens, offsets (None: n_q each), n_q, causal, mask
    ("bf16", 64, 2, 4, [300], None, 1, True, None),
    ("f16", 128, 2, 4, [1, 63, 64, 65, 0, 127, 500], None, 1, True, None),
    ("bf16", 96, 3, 5, [200, 513, 70], None, 3, True, None),
    ("f16", 256, 1, 1, [700, 3], None, 2, False, None),
    ("bf16", 128, 2, 2, [1030, 64], None, 37, False, None),
    ("f16", 64, 1, 16, [257, 130], None, 2, True, "half"),
    ("bf16", 128, 1, 20, [90, 640], None, 1, True, "sparse"),
    ("bf16", 96, 2, 1, [400, 90, 1], [0, 17, 17, 18], 0, True, None),
    ("f16", 128, 2, 3, [100, 333, 64, 0], [0, 65, 70, 70, 75], 0, True, "half"),
    ("bf16", 256, 2, 8, [2100], None, 19, True, "sparse"),
    ("f16", 64, 1, 1, [5], None, 9, True, None),  # more tokens than the sequence holds: rows that see nothing
    ("bf16", 128, 1, 4, [9000], None, 1, True, None),
    ("f16", 96, 1, 2, [130, 2000], None, 150, True, None),
    ("bf16", 64, 2, 4, [1500, 77], None, 130, True, "half"),
]


@pytest.mark.parametrize("with_mass", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention_matches_plain(case, with_mass):
    dtype, d, heads, group, lens, offsets, n_q, causal, kind = CASES[case]
    say(f"[kv] attend case {case}: {CASES[case]} mass={with_mass}")
    rng = np.random.default_rng(100 + case)
    host = R.Host(rng, lens, heads, d, max_blocks=-(-max(lens) // 64) + 2)
    n_tok = offsets[-1] if offsets else n_q * len(lens)
    q = queries(rng, n_tok, heads * group, d, dtype)
    mask = masks(rng, n_tok, host.max_blocks, kind)
    mass = rng.uniform(0, 3, (len(lens), heads, host.max_blocks)).astype(np.float32) if with_mass else None
    kw = {"max_tok": max(np.diff(offsets)).item()} if offsets else {}
    cache, batch = host.cache(st), host.batch(st, n_tok, offsets, max_len=max(lens), **kw)
    lse = torch.full((n_tok, heads * group), 7.0, device="cuda")
    out = torch.full((n_tok, heads * group, d), 7.0, dtype=TYPES[dtype], device="cuda")
    mass_out = torch.full((len(lens), heads, host.max_blocks), 7.0, device="cuda") if with_mass else None
    args = dict(causal=causal, mask=cuda_mask(mask), lse=lse, out=out, decay=0.75, mass_out=mass_out,
                mass=None if mass is None else torch.from_numpy(mass).cuda())
    st.st_kv_attend(cache, batch, q.cuda(), **args)
    torch.cuda.synchronize()
    want, want_lse, want_mass, reach = R.attend(host, q, d ** -0.5, causal, offsets, mask, None, mass, 0.75)
    check_out(out, want, reach, host, dtype)
    got_lse = lse.cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isinf(got_lse), np.isinf(want_lse)) and np.all(got_lse[np.isinf(want_lse)] < 0)
    fin = np.isfinite(want_lse)
    tol = (2 * (d + 8) * reach + max(lens) / 16 + 64 + 4 * np.abs(np.where(fin, want_lse, 0))) * 2.0 ** -23
    assert np.all(np.abs(got_lse - want_lse)[fin] <= tol[fin])
    if with_mass:
        rows = n_q * group if not offsets else max(np.diff(offsets)) * group
        rel = (4 * (d + 8) * reach.max(initial=0) + max(lens) / 8 + 128 + rows) * 2.0 ** -23
        got = mass_out.cpu().numpy()
        assert np.all(np.abs(got - want_mass) <= rel * rows + 2.0 ** -22 * want_mass + 1e-30)
    # the same call again gives the same bits
    again = out.clone(), lse.clone()
    st.st_kv_attend(cache, batch, q.cuda(), **args)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)


SELECTS = [
    # dtype, d, heads, group, lens, offsets, n_q, causal, mask, n_sel, sink, recent
    ("bf16", 64, 2, 4, [1200], None, 1, True, None, 6, 1, 2),
    ("f16", 128, 2, 2, [640, 5000, 1, 0, 64], None, 1, True, None, 9, 0, 0),
    ("bf16", 96, 3, 5, [2000, 700], None, 5, True, None, 4, 0, 1),
    ("f16", 256, 1, 1, [3000], None, 18, False, "sparse", 7, 2, 1),
    ("bf16", 128, 2, 1, [900, 300], [0, 33, 35], 0, False, "half", 5, 0, 0),
    ("f16", 64, 1, 20, [20000], None, 1, True, None, 40, 3, 5),
    ("bf16", 128, 1, 8, [500], None, 2, True, None, 100, 1, 1),  # more than there are
]


@pytest.mark.parametrize("case", range(len(SELECTS)))
def test_selection_and_attention_over_it_match_plain(case):
    dtype, d, heads, group, lens, offsets, n_q, causal, kind, n_sel, sink, recent = SELECTS[case]
    say(f"[kv] select case {case}: {SELECTS[case]}")
    rng = np.random.default_rng(200 + case)
    host = R.Host(rng, lens, heads, d)
    n_tok = offsets[-1] if offsets else n_q * len(lens)
    q = queries(rng, n_tok, heads * group, d, dtype)
    mask = masks(rng, n_tok, host.max_blocks, kind)
    cache, batch = host.cache(st), host.batch(st, n_tok, offsets)
    blocks = st.st_kv_select(cache, batch, q.cuda(), n_sel, causal=causal, mask=cuda_mask(mask), sink=sink, recent=recent)
    torch.cuda.synchronize()
    want = R.select(host, q, n_sel, causal, sink, recent, offsets, mask)
    assert np.array_equal(blocks.cpu().numpy(), want)
    mass = rng.uniform(0, 3, (len(lens), heads, host.max_blocks)).astype(np.float32)
    mass_out = torch.full(mass.shape, 7.0, device="cuda")
    out = st.st_kv_attend(cache, batch, q.cuda(), causal=causal, mask=cuda_mask(mask), blocks=blocks, decay=0.5,
                          mass=torch.from_numpy(mass).cuda(), mass_out=mass_out)
    torch.cuda.synchronize()
    ref, _, ref_mass, reach = R.attend(host, q, d ** -0.5, causal, offsets, mask, want, mass, 0.5)
    check_out(out, ref, reach, host, dtype)
    rows = n_tok * group
    rel = (4 * (d + 8) * reach.max(initial=0) + max(lens) / 8 + 128 + rows) * 2.0 ** -23
    assert np.all(np.abs(mass_out.cpu().numpy() - ref_mass) <= rel * rows + 2.0 ** -22 * ref_mass + 1e-30)


def test_equal_scores_go_to_the_lower_block_and_zero_queries_select():
    rng = np.random.default_rng(3)
    host = R.Host(rng, [64 * 300, 64 * 40], 1, 64)
    host.bounds[:] = 5
    host.ks[:] = np.float32(0.25)
    host.k[:] = 5
    q = queries(rng, 2, 1, 64, "bf16")
    q[1] = 0
    got = st.st_kv_select(host.cache(st), host.batch(st, 2), q.cuda(), 21, sink=2, recent=3)
    assert np.array_equal(got.cpu().numpy(), R.select(host, q, 21, True, 2, 3))
    assert got[1, 0].tolist() == list(range(18)) + [37, 38, 39]


def test_lists_in_any_order_and_out_of_range_entries():
    rng = np.random.default_rng(4)
    host = R.Host(rng, [1000, 400], 2, 128)
    q = queries(rng, 2, 4, 128, "f16")
    blocks = np.array([[[9, -5, 3, 0, 400], [15, 14, 1, 16, -1]], [[6, 2, -1, -1, 7], [-1, -1, -1, -1, -1]]], np.int32)
    out = st.st_kv_attend(host.cache(st), host.batch(st, 2), q.cuda(), blocks=torch.from_numpy(blocks).cuda())
    ref, _, _, reach = R.attend(host, q, 128 ** -0.5, True, None, None, blocks)
    check_out(out, ref, reach, host, "f16")
    assert out[1, 2:].abs().max() == 0


def test_pages_out_of_range_count_as_masked_and_lengths_are_cut():
    rng = np.random.default_rng(5)
    host = R.Host(rng, [640, 300], 1, 64)
    q = queries(rng, 2, 2, 64, "bf16")
    cache, batch = host.cache(st), host.batch(st, 2, max_len=576)
    batch.tables[0, 3], batch.tables[0, 7], batch.tables[1, 0] = 1 << 30, -7, cache.n_pages
    out = st.st_kv_attend(cache, batch, q.cuda())
    host.lens = [576, 300]
    blocks = np.array([[[0, 1, 2, 4, 5, 6, 8]], [[1, 2, 3, 4, -1, -1, -1]]], np.int32)
    ref, _, _, reach = R.attend(host, q, 64 ** -0.5, True, None, None, blocks)
    check_out(out, ref, reach, host, "bf16")
    chosen = st.st_kv_select(cache, batch, q.cuda(), 20).cpu().numpy()
    assert chosen[0, 0, :9].tolist() == [0, 1, 2, 4, 5, 6, 8, -1, -1] and chosen[1, 0, :5].tolist() == [1, 2, 3, 4, -1]


@pytest.mark.parametrize("size", [1e-30, 30.0, 3000.0])
def test_queries_of_extreme_size(size):
    rng = np.random.default_rng(6)
    host = R.Host(rng, [700], 2, 128)
    q = queries(rng, 4, 4, 128, "bf16", size)
    out = st.st_kv_attend(host.cache(st), host.batch(st, 4), q.cuda())
    ref, _, _, reach = R.attend(host, q, 128 ** -0.5, True)
    check_out(out, ref, reach, host, "bf16")


def test_not_a_number_stays_in_its_row():
    rng = np.random.default_rng(7)
    host = R.Host(rng, [900], 1, 64)
    q = queries(rng, 5, 3, 64, "bf16")
    clean = st.st_kv_attend(host.cache(st), host.batch(st, 5), q.cuda(), causal=False)
    q[2, 1, 5] = float("nan")
    out = st.st_kv_attend(host.cache(st), host.batch(st, 5), q.cuda(), causal=False)
    assert out[2, 1].isnan().all()
    out[2, 1], clean[2, 1] = 0, 0
    assert torch.equal(out, clean)


MANY = [  # tiles of 256 (d = 256: 128) rows, whole and cut short, with and without splits
    ("bf16", 128, 2, 2, [1030, 64], None, 150, False, None),
    ("f16", 96, 1, 5, [640, 2000, 0, 333], [0, 60, 130, 130, 131], 0, True, "half"),
    ("bf16", 64, 1, 1, [5, 400], None, 300, True, None),
    ("f16", 256, 1, 3, [700, 130], None, 100, True, "sparse"),
    ("bf16", 256, 2, 4, [130, 1], None, 70, False, None),
    ("f16", 128, 1, 4, [4000], None, 80, True, "sparse"),
    ("bf16", 96, 3, 1, [64, 65, 150], None, 257, False, "half"),
]


@pytest.mark.parametrize("with_mass", [False, True])
@pytest.mark.parametrize("case", range(len(MANY)))
def test_many_rows_match_plain(case, with_mass, monkeypatch):
    monkeypatch.setitem(globals(), "CASES", MANY)
    test_attention_matches_plain(case, with_mass)


@pytest.mark.parametrize("d", [64, 256])
def test_not_a_number_stays_in_its_row_of_many(d):
    rng = np.random.default_rng(27)
    host = R.Host(rng, [900], 1, d)
    q = queries(rng, 100, 3, d, "bf16")
    clean = st.st_kv_attend(host.cache(st), host.batch(st, 100), q.cuda(), causal=False)
    q[2, 1, 5], q[99, 2, 0] = float("nan"), float("inf")
    out = st.st_kv_attend(host.cache(st), host.batch(st, 100), q.cuda(), causal=False)
    for row in ((2, 1), (99, 2)):
        assert out[row].isnan().all()
        out[row], clean[row] = 0, 0
    assert torch.equal(out, clean)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("group", [1, 4])
def test_not_a_number_stays_in_its_row_of_few(group, bad):
    rng = np.random.default_rng(17)
    host = R.Host(rng, [900, 200], 2, 128)
    q = queries(rng, 2, 2 * group, 128, "f16")
    clean = st.st_kv_attend(host.cache(st), host.batch(st, 2), q.cuda())
    q[1, group, 77] = bad
    out = st.st_kv_attend(host.cache(st), host.batch(st, 2), q.cuda())
    assert out[1, group].isnan().all()
    out[1, group], clean[1, group] = 0, 0
    assert torch.equal(out, clean)


@pytest.mark.parametrize("n_q,group", [(1, 1), (1, 4), (2, 2), (4, 1)])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_up_to_four_rows(n_q, group, d):
    """Few rows: one large weight among many small ones, values of one sign."""
    rng = np.random.default_rng(18 + d)
    lens = [64 * 30 + 7, 500, 3]
    host = R.Host(rng, lens, 2, d)
    host.v = np.abs(host.v.astype(np.int32)).clip(0, 127).astype(np.int8)
    n_tok = n_q * len(lens)
    q = queries(rng, n_tok, 2 * group, d, "f16", 0.01)
    for s, n in enumerate(lens):  # the first row of each sequence finds one key 11 nats above the others
        page, at = host.tables[s, n // 2 // 64], n // 2 % 64
        key = host.k[page, 0, at].astype(np.float64) * host.ks[page, 0]
        q[s * n_q, 0] = torch.from_numpy(11 * d ** 0.5 * key / (key @ key)).half()
    lse = torch.zeros((n_tok, 2 * group), device="cuda")
    out = st.st_kv_attend(host.cache(st), host.batch(st, n_tok), q.cuda(), causal=False, lse=lse)
    want, want_lse, _, reach = R.attend(host, q, d ** -0.5, False)
    check_out(out, want, reach, host, "f16")
    tol = (2 * (d + 8) * reach + max(lens) / 16 + 64 + 4 * np.abs(want_lse)) * 2.0 ** -23
    assert np.all(np.abs(lse.cpu().numpy() - want_lse) <= tol)


def test_rows_inside_wider_rows():
    rng = np.random.default_rng(8)
    host = R.Host(rng, [300, 200], 2, 64)
    wide = queries(rng, 6, 12, 64, "bf16").cuda()
    q = wide[:, 4:8]
    a = st.st_kv_attend(host.cache(st), host.batch(st, 6), q)
    b = st.st_kv_attend(host.cache(st), host.batch(st, 6), q.contiguous())
    assert torch.equal(a, b)
    c1, c2 = host.cache(st), host.cache(st)
    k, v = wide[:, 8:10], wide[:, 10:12]
    st.st_kv_append(c1, host.batch(st, 6), k, v)
    st.st_kv_append(c2, host.batch(st, 6), k.contiguous(), v.contiguous())
    assert all(torch.equal(x, y) for x, y in ((c1.k, c2.k), (c1.v, c2.v), (c1.bounds, c2.bounds)))
    assert torch.equal(st.st_kv_select(c1, host.batch(st, 6), q, 3), st.st_kv_select(c1, host.batch(st, 6), q.contiguous(), 3))


def same_tokens(host, cache, touched=None):
    """Integers, scales and bounds of every position that holds a token."""
    v = cache.v.cpu().numpy()[..., R.SLOTS].swapaxes(2, 3)
    k = cache.k.cpu().numpy()
    for s, n in enumerate(host.lens):
        for b in range(-(-n // 64)):
            p, m = host.tables[s, b], min(64, n - 64 * b)
            assert np.array_equal(k[p, :, :m], host.k[p, :, :m]), (s, b)
            assert np.array_equal(v[p, :, :m], host.v[p, :, :m]), (s, b)
            for got, want in ((cache.k_scale, host.ks), (cache.v_scale, host.vs)):
                assert np.array_equal(got[p].cpu().numpy().view(np.uint32), want[p].view(np.uint32)), (s, b)
            assert np.array_equal(cache.bounds[p].cpu().numpy(), host.bounds[p]), (s, b)


@pytest.mark.parametrize("dtype,d,heads,before,new", [
    ("bf16", 64, 2, [0, 63, 64, 65, 100], 1), ("f16", 128, 1, [0, 1, 130], 3), ("bf16", 96, 3, [10, 0], 200),
    ("f16", 256, 2, [5, 64], 64), ("bf16", 128, 8, [0], 1), ("f16", 96, 1, [31, 32, 95], [0, 1, 1, 78])])
def test_appends_match_plain(dtype, d, heads, before, new):
    say(f"[kv] append {dtype} d={d} before={before} new={new}")
    rng = np.random.default_rng(d + heads)
    offsets = None if isinstance(new, int) else new
    counts = [new] * len(before) if offsets is None else list(np.diff(new))
    host = R.Host(rng, before, heads, d, spare=40, max_blocks=8)
    cache = host.cache(st)
    spare = [p for p in range(len(host.k)) if p not in host.tables]
    held = [-(-n // 64) for n in before]
    for round_ in range(4):  # growing sizes: the blocks' scales grow with them; then smaller ones
        host.lens = [n + c for n, c in zip(host.lens, counts)]
        for s, n in enumerate(host.lens):
            while held[s] < -(-n // 64) and held[s] < 8:
                host.tables[s, held[s]] = spare.pop()
                held[s] += 1
        if max(host.lens) > 8 * 64:
            break
        n_tok = sum(counts)
        rows = [queries(rng, n_tok, heads, d, dtype, (0.2, 3.0, 10.0, 0.0)[round_]) for _ in range(2)]
        kw = {} if offsets is None else {"max_tok": max(counts)}
        batch = host.batch(st, n_tok, offsets, **kw)
        st.st_kv_append(cache, batch, rows[0].cuda(), rows[1].cuda())
        R.append(host, *rows, offsets)
        same_tokens(host, cache)
        st.st_kv_append(cache, batch, rows[0].cuda(), rows[1].cuda())  # again: nothing changes
        same_tokens(host, cache)
        k, v, bounds = (x.cpu().numpy() for x in st.st_kv_read(cache, batch, 3))
        for s, n in enumerate(host.lens):
            first = max(0, held[s] - 3)
            for j in range(3):
                m = max(0, min(64, n - 64 * (first + j)))
                assert not k[s, j, :, m:].any() and not v[s, j, :, m:].any()
                if m:
                    p = host.tables[s, first + j]
                    assert np.array_equal(k[s, j, :, :m], host.k[p, :, :m].astype(np.float32) * host.ks[p][:, None, None])
                    assert np.array_equal(v[s, j, :, :m], host.v[p, :, :m].astype(np.float32) * host.vs[p][:, None, None])
                    assert np.array_equal(bounds[s, j], host.bounds[p].astype(np.float32) * host.ks[p][:, None, None])
                else:
                    assert not bounds[s, j].any()


def test_append_skips_what_has_no_place():
    rng = np.random.default_rng(9)
    host = R.Host(rng, [200, 100], 1, 64, max_blocks=6)
    cache = host.cache(st)
    batch = host.batch(st, 260)  # 130 tokens each: the second sequence holds 100, so 30 come before its position 0
    batch.tables[0, 2] = 1 << 20
    before = cache.k.clone(), cache.k_scale.clone()
    rows = [queries(rng, 260, 1, 64, "bf16") for _ in range(2)]
    st.st_kv_append(cache, batch, rows[0].cuda(), rows[1].cuda())
    skipped = host.tables[0, 2]
    host.tables[0, 2] = 1 << 20
    R.append(host, *rows)
    host.tables[0, 2] = skipped
    same_tokens(host, cache)
    written = set(host.tables[host.tables >= 0]) - {skipped}
    for p in range(cache.n_pages):
        if p not in written:
            assert torch.equal(cache.k[p], before[0][p]) and torch.equal(cache.k_scale[p].isnan(), before[1][p].isnan())


@pytest.mark.parametrize("lens,heads,budget,sink,recent", [
    ([5000], 2, 40, 1, 2), ([64 * 700 + 1, 0, 1, 64, 30000], 3, 100, 4, 8), ([6400, 6401], 1, 1, 0, 1), ([640], 8, 500, 3, 3),
    ([64 * 2000], 2, 1999, 0, 1)])
def test_evictions_match_plain(lens, heads, budget, sink, recent):
    rng = np.random.default_rng(sum(lens))
    held = [-(-n // 64) for n in lens]
    nb = max(held) + 3
    tables = np.full((len(lens), nb), -1, np.int32)
    order = rng.permutation(sum(held))
    for s in range(len(lens)):
        tables[s, : held[s]] = order[sum(held[:s]): sum(held[: s + 1])]
    mass = np.round(rng.uniform(0, 1, (len(lens), heads, nb)) ** 6, 2).astype(np.float32)  # with many equal ones
    want = R.evict(tables, lens, mass, budget, sink, recent)
    t, n, m = torch.from_numpy(tables).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), torch.from_numpy(mass).cuda()
    batch = st.KvBatch(t, n, 0)
    got = st.st_kv_evict(batch, m, budget, sink=sink, recent=recent)
    for g, w in zip(got, want):
        assert np.array_equal(g.cpu().numpy(), w)
    st.st_kv_evict(batch, m, budget, sink=sink, recent=recent, out=(t, n, m, got[3], got[4]))  # in place
    for g, w in zip((t, n, m, got[3], got[4]), want):
        assert np.array_equal(g.cpu().numpy(), w)


def test_on_a_stream_of_its_own_and_captured():
    rng = np.random.default_rng(11)
    host = R.Host(rng, [3000, 700], 2, 128)
    q = queries(rng, 2, 8, 128, "bf16").cuda()
    new = queries(rng, 2, 2, 128, "bf16").cuda()
    cache, batch = host.cache(st), host.batch(st, 2)
    buf = st.KvBuffers(cache, batch, q, n_sel=8, mass=True)
    mass = torch.rand((2, 2, host.max_blocks), device="cuda")
    kept = st.st_kv_evict(batch, mass, 20)

    def step():
        st.st_kv_append(cache, batch, new, new)
        blocks = st.st_kv_select(cache, batch, q, 8, sink=1, recent=1, buffers=buf)
        st.st_kv_attend(cache, batch, q, blocks=blocks, mass=mass, buffers=buf)
        st.st_kv_evict(batch, buf.mass, 20, out=kept)

    step()
    want = [x.clone() for x in (buf.out, buf.mass, buf.blocks, *kept)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for x in (buf.out, buf.mass, buf.blocks, *kept):
            x.zero_()
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, (buf.out, buf.mass, buf.blocks, *kept)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):  # replays with other queries, eager work between them
        q.copy_(torch.roll(q, 1, 2))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (buf.out, buf.mass, buf.blocks, *kept)]
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, (buf.out, buf.mass, buf.blocks, *kept))), f"replay {i}"


def test_offsets_into_the_cache_pass_32_bits():
    # pages beyond 2^32 bytes of keys: 140,000 pages of 4 heads x 64 x 128 integers
    say("[kv] a cache of 4.6 GB for keys and as much for values")
    n_pages, heads, d = 140_000, 4, 128
    cache = st.KvCache.empty(n_pages, heads, d)
    rng = np.random.default_rng(12)
    host = R.Host(rng, [640, 100], heads, d, spare=0)
    far = n_pages - 1 - np.arange(len(host.k))
    small = host.cache(st)
    for name in ("k", "v", "k_scale", "v_scale", "bounds"):
        getattr(cache, name)[torch.from_numpy(far.copy()).cuda()] = getattr(small, name)
    tables = np.where(host.tables >= 0, far[np.maximum(host.tables, 0)], -1).astype(np.int32)
    q = queries(rng, 2, 8, d, "bf16").cuda()
    a, b = host.batch(st, 2), host.batch(st, 2)
    b.tables.copy_(torch.from_numpy(tables))
    assert torch.equal(st.st_kv_attend(small, a, q), st.st_kv_attend(cache, b, q))
    assert torch.equal(st.st_kv_select(small, a, q, 4), st.st_kv_select(cache, b, q, 4))
    new = queries(rng, 2, heads, d, "bf16").cuda()
    st.st_kv_append(small, a, new, new)
    st.st_kv_append(cache, b, new, new)
    for x, y in zip(st.st_kv_read(small, a, 2), st.st_kv_read(cache, b, 2)):
        assert torch.equal(x, y)


def test_empty_calls():
    host = R.Host(np.random.default_rng(13), [100], 1, 64)
    cache = host.cache(st)
    none = torch.zeros((0, 4), dtype=torch.int32, device="cuda")
    batch = st.KvBatch(none, none[:, 0].contiguous(), 0)
    q = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    assert st.st_kv_attend(cache, batch, q).shape == (0, 2, 64)
    assert st.st_kv_select(cache, batch, q, 3).shape == (0, 1, 3)
    st.st_kv_append(cache, batch, q[:, :1], q[:, :1])
    mass = torch.rand((1, 1, 2), device="cuda")
    out = torch.zeros_like(mass)
    none_new = host.batch(st, 0)
    st.st_kv_attend(cache, none_new, q, mass=mass, decay=0.5, mass_out=out)  # no tokens: the weights decay
    assert torch.equal(out, mass * 0.5)
