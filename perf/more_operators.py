"""Timed cases of the operators of a layer around the cached histories: the norm that turns rows into int8, the
projection of int8 rows with low-rank adapters of many requests, rotary positions with several axes, and the copying of
the cache's pages.

``run`` makes the calls of ``paper_2511_14881_amd.binding`` where ``own`` is true and computes the same in
elementary torch operations otherwise.  Heads and widths of a head are those of the cached histories (64, 96, 128), 500
candidates for each of 16 users those of the attention over them; model widths and numbers of rows are generic.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 64
_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_NORM_VALUES = 65_536 * 2048           # of the largest norm
_PROJECT_WORK = 3.6e11                 # multiply-adds of the largest projection
_ROTATE_VALUES = 32_768 * 40 * 128     # of the largest rotation
_COPY_BYTES = 2048 * 8 * 128 * 128     # of the largest copy's keys and values


def _norm(name, *, rows, d, dtype="bf16", residual=True, y=False):
    case = {"op": "norm", "rows": rows, "d": d, "dtype": dtype, "residual": residual, "y": y}
    return {**case, "name": name} if name else case


def _project(name, *, rows, k, n, adapters=0, rank=16, mixed=False, dtype="bf16"):
    case = {"op": "project", "rows": rows, "k": k, "n": n, "adapters": adapters, "rank": rank, "mixed": mixed, "dtype": dtype}
    return {**case, "name": name} if name else case


def _rotate(name, *, tokens, heads, kv_heads, d, axes, part=1.0, interleaved=False, dtype="bf16"):
    case = {"op": "rotate", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "d": d, "axes": axes, "part": part,
            "interleaved": interleaved, "dtype": dtype}
    return {**case, "name": name} if name else case


def _copy(name, *, copies, heads, d):
    case = {"op": "copy", "copies": copies, "heads": heads, "d": d}
    return {**case, "name": name} if name else case


def listed():
    return [
        # one user's newest event, a narrow layer: a launch and its latency
        _norm("norm-1", rows=1, d=256),
        # 500 candidates for each of 16 users, a width that is no power of two; the norm's output in 16 bits too
        _norm("norm-candidates", rows=8000, d=1008, dtype="f16", residual=False, y=True),
        # histories taken in from the log: bandwidth
        _norm("norm-events", rows=65_536, d=2048),
        # one event to queries, keys and values, with the adapter of its market
        _project("project-1", rows=1, k=512, n=1024, adapters=8),
        # an online batch: an event for each of 64 users, adapters in no order: the weights' bytes
        _project("project-64", rows=64, k=4096, n=5120, adapters=32, mixed=True),
        # candidates of odd counts and widths, small adapters in no order
        _project("project-candidates", rows=1001, k=1040, n=1296, adapters=5, rank=8, mixed=True, dtype="f16"),
        # histories taken in from the log, request after request: the int8 products
        _project("project-events", rows=16_384, k=4096, n=5120, adapters=16, rank=32),
        # one event: queries of 4 heads, keys of 1
        _rotate("rotate-1", tokens=1, heads=4, kv_heads=1, d=64, axes=2),
        # candidates with an index and a time, three quarters of a row rotated, neighbouring pairs
        _rotate("rotate-candidates", tokens=8000, heads=8, kv_heads=2, d=128, axes=2, part=0.75, interleaved=True, dtype="f16"),
        # histories taken in from the log, with index, time and session
        _rotate("rotate-events", tokens=32_768, heads=32, kv_heads=8, d=128, axes=3),
        # a history is forked: its last page is copied
        _copy("copy-1", copies=1, heads=2, d=64),
        # a cache is compacted
        _copy("copy-2048", copies=2048, heads=8, d=128),
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["norm", "project", "project", "project", "rotate", "rotate", "copy"])
    dtype = rng.choice(["bf16", "f16"])
    if op == "norm":
        d = 16 * _log(rng, 2, 512)
        rows = min(_log(rng, 1, 65_536), _NORM_VALUES // d)
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        if dtype == "f32":
            rows = max(1, rows // 2)
        return _norm(None, rows=rows, d=d, dtype=dtype, residual=rng.random() < 0.7, y=rng.random() < 0.3)
    if op == "project":
        k, n = 16 * _log(rng, 4, 512), 16 * _log(rng, 4, 512)
        adapters, rank = rng.choice([0, 1, _log(rng, 2, 64), _log(rng, 2, 64)]), rng.choice([8, 16, 16, 32, 64, 128])
        each = k * n + adapters * rank * (k + n)
        rows = max(1, min(_log(rng, 1, 16_384), int(_PROJECT_WORK / each)))
        return _project(None, rows=rows, k=k, n=n, adapters=adapters, rank=rank, mixed=rng.random() < 0.5, dtype=dtype)
    if op == "rotate":
        kv_heads, d = rng.choice([1, 2, 3, 4, 8]), rng.choice([64, 96, 128, 128, 256])
        heads = kv_heads * rng.choice([1, 2, 4, 5])
        tokens = min(_log(rng, 1, 32_768), _ROTATE_VALUES // ((heads + kv_heads) * d))
        return _rotate(None, tokens=tokens, heads=heads, kv_heads=kv_heads, d=d, axes=rng.choice([1, 2, 3]),
                       part=rng.choice([0.5, 1.0, 1.0]), interleaved=rng.random() < 0.5, dtype=dtype)
    heads, d = rng.choice([1, 2, 3, 4, 8]), rng.choice([64, 96, 128, 256])
    return _copy(None, copies=min(_log(rng, 1, 4096), _COPY_BYTES // (heads * d * 2 * BLOCK)), heads=heads, d=d)


def _sections(case):
    """Pairs of each axis: the first has the most."""
    pairs = int(case["d"] * case["part"]) // 16 * 8
    rest = pairs // (case["axes"] + 1)
    return [pairs - rest * (case["axes"] - 1)] + [rest] * (case["axes"] - 1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    state = {"case": dict(case), "kept": {}}
    if case["op"] == "norm":
        rows, d, dtype = case["rows"], case["d"], _TYPES[case["dtype"]]
        # channels differ in size, some by much, and so do rows
        size = torch.exp(normal(d) * 0.5) * torch.where(torch.rand(d, generator=gen, device="cuda") < 0.01, 12.0, 1.0)
        state["x"] = (normal(rows, d) * size * torch.exp(normal(rows, 1) * 0.5)).to(dtype)
        state["weight"] = (1.0 + 0.2 * normal(d)).to(dtype)
        if case["residual"]:
            state["residual"] = (normal(rows, d) * size).to(dtype)
        return state
    if case["op"] == "project":
        rows, k, n, count, rank, dtype = case["rows"], case["k"], case["n"], case["adapters"], case["rank"], _TYPES[case["dtype"]]
        state["x"] = (normal(rows, k) * 36.0).round().clamp(-127, 127).to(torch.int8)
        state["x_scale"] = torch.exp(normal(rows) * 0.3) / 36.0
        state["w"] = (normal(n, k) * 36.0).round().clamp(-127, 127).to(torch.int8)
        state["w_scale"] = torch.exp(normal(n) * 0.3) / (36.0 * math.sqrt(k))
        if count:
            state["a"] = (normal(count, rank, k) / math.sqrt(k)).to(dtype)
            state["b"] = (normal(count, n, rank) * 0.3).to(dtype)
            state["alpha"] = (1.0 + torch.rand(count, generator=gen, device="cuda")) / math.sqrt(rank)
            # requests one behind the other, or mixed; one row in 16 of the mixed ones has no adapter
            at = torch.arange(rows, device="cuda") * count // rows
            if case["mixed"]:
                at = torch.randint(0, count, (rows,), generator=gen, device="cuda")
                at[torch.rand(rows, generator=gen, device="cuda") < 1 / 16] = -1
            state["adapter_of"] = at.to(torch.int32)
        return state
    if case["op"] == "rotate":
        tokens, heads, kv_heads, d, dtype = case["tokens"], case["heads"], case["kv_heads"], case["d"], _TYPES[case["dtype"]]
        # queries, keys and values lie side by side, as a projection writes them
        qkv = normal(tokens, heads + 2 * kv_heads, d).to(dtype)
        state["q"], state["k"] = qkv[:, :heads], qkv[:, heads:heads + kv_heads]
        index = torch.arange(tokens, device="cuda") % 5000
        time = 1_700_000_000 + torch.randint(0, 40_000_000, (tokens,), generator=gen, device="cuda")
        session = torch.randint(0, 400, (tokens,), generator=gen, device="cuda")
        state["positions"] = torch.stack([index, time, session][:case["axes"]]).to(torch.int32)
        freqs = []
        for axis, count in enumerate(_sections(case)):
            turn = torch.arange(count, device="cuda", dtype=torch.float64) / count
            # an index: 1 to 1 / 10000; a time in seconds: periods from a minute to ten years; a session: as an index
            freqs.append(2 * math.pi / 60.0 * (60.0 / 3.2e8) ** turn if axis == 1 else 10_000.0 ** -turn)
        state["freqs"] = torch.cat(freqs)
        return state
    copies, heads, d = case["copies"], case["heads"], case["d"]
    pages = 2 * copies + 3
    order = torch.randperm(pages, generator=gen, device="cuda", dtype=torch.int32)
    state["src"], state["dst"] = order[:copies].clone(), order[copies:2 * copies].clone()

    def integers(*shape):
        return torch.randint(-127, 128, shape, generator=gen, device="cuda", dtype=torch.int8)

    state.update(k=integers(pages, heads, BLOCK, d), v=integers(pages, heads, d, BLOCK), bounds=integers(pages, heads, 2, d),
                 k_scale=torch.rand((pages, heads), generator=gen, device="cuda"),
                 v_scale=torch.rand((pages, heads), generator=gen, device="cuda"))
    return state


# ---------------------------------------------------------------------------------------- the framework's calls


def _run_own(state):
    from paper_2511_14881_amd import binding as st

    case, kept = state["case"], state["kept"]
    if case["op"] == "norm":
        if not kept:  # what a program makes once and keeps: outputs
            kept["buffers"] = st.RowBuffers(case["rows"], case["d"], _TYPES[case["dtype"]], total=case["residual"], y=case["y"])
        got = st.st_norm_rows(state["x"], state["weight"], state.get("residual"), buffers=kept["buffers"])
        values = got.q * got.scale[:, None]
        return [values] + ([got.total] if case["residual"] else []) + ([got.y] if case["y"] else [])
    if case["op"] == "project":
        adapters = None
        if not kept:  # the adapters' handle, output and workspace
            if case["adapters"]:
                kept["adapters"] = st.Adapters(state["a"], state["b"], state["alpha"])
            kept["buffers"] = st.ProjectBuffers(case["rows"], case["k"], case["n"], _TYPES[case["dtype"]], kept.get("adapters"))
        adapters = kept.get("adapters")
        return st.st_project(state["x"], state["x_scale"], state["w"], state["w_scale"], adapters, state.get("adapter_of"),
                             buffers=kept["buffers"])
    if case["op"] == "rotate":
        if not kept:
            kept["out"] = torch.empty_like(state["q"]), torch.empty_like(state["k"])
        return st.st_rotate(state["q"], state["k"], state["positions"], state["freqs"], _sections(case),
                            interleaved=case["interleaved"], out=kept["out"])
    if not kept:
        kept["cache"] = st.KvCache(state["k"], state["v"], state["k_scale"], state["v_scale"], state["bounds"])
    st.st_kv_copy(kept["cache"], kept["cache"], state["src"], state["dst"])
    return [state[name] for name in ("k", "v", "k_scale", "v_scale", "bounds")]


# ---------------------------------------------------------------------------------------- the plain forms


def _run_norm(state):
    case, x = state["case"], state["x"]
    total = (x.float() + state["residual"].float()).to(x.dtype) if case["residual"] else x
    h = total.float()
    t = h * state["weight"].float()
    unit = t.abs().amax(-1, keepdim=True)
    unit = unit / torch.full_like(unit, 127.0)
    q = torch.where(unit > 0, torch.round(t / unit), torch.zeros_like(t)).clamp(-127, 127)
    rms = 1.0 / torch.sqrt(h.square().mean(-1, keepdim=True) + 1e-6)
    values = q * (unit * rms)
    return [values] + ([total] if case["residual"] else []) + ([(t * rms).to(x.dtype)] if case["y"] else [])


def _run_project(state):
    case = state["case"]
    count, rank = case["adapters"], case["rank"]
    x = state["x"].float()
    out = torch.matmul(x, state["w"].float().t()) * state["x_scale"][:, None] * state["w_scale"]
    if count:
        # all adapters' inner values, of which each row keeps its own
        inner = torch.matmul(x, state["a"].float().flatten(0, 1).t()).view(-1, count, rank)
        mine = state["adapter_of"][:, None] == torch.arange(count, device="cuda")
        inner = torch.where(mine[..., None], inner * state["alpha"][:, None], torch.zeros_like(inner))
        outer = state["b"].float().transpose(1, 2).reshape(count * rank, -1)
        out = out + torch.matmul(inner.flatten(1), outer) * state["x_scale"][:, None]
    return out.to(_TYPES[case["dtype"]])


def _run_rotate(state):
    case = state["case"]
    sections = torch.tensor(_sections(case), device="cuda")
    axis = torch.repeat_interleave(torch.arange(case["axes"], device="cuda"), sections, output_size=state["freqs"].numel())
    angle = state["positions"].t()[:, axis].double() * state["freqs"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    pairs = angle.shape[1]

    def turned(rows):
        x = rows[..., :2 * pairs].float()
        a, b = (x[..., 0::2], x[..., 1::2]) if case["interleaved"] else (x[..., :pairs], x[..., pairs:])
        a, b = a * cos - b * sin, a * sin + b * cos
        x = torch.stack([a, b], -1).flatten(-2) if case["interleaved"] else torch.cat([a, b], -1)
        return torch.cat([x.to(rows.dtype), rows[..., 2 * pairs:]], -1)

    return turned(state["q"]), turned(state["k"])


def _run_copy(state):
    src, dst = state["src"].long(), state["dst"].long()
    names = ("k", "v", "k_scale", "v_scale", "bounds")
    for name in names:
        state[name][dst] = state[name][src]
    return [state[name] for name in names]


def run(state):
    if own:
        return _run_own(state)
    return {"norm": _run_norm, "project": _run_project, "rotate": _run_rotate, "copy": _run_copy}[state["case"]["op"]](state)


def work(case):
    """Each input read once and each output written once; two operations to a multiply and add."""
    if case["op"] == "norm":
        size = 4 if case["dtype"] == "f32" else 2
        values = case["rows"] * case["d"]
        arrays = 1 + 2 * case["residual"] + case["y"]  # of the type: rows, residual and sum, the norm's output
        return {"bytes": values * (size * arrays + 4) + size * case["d"], "flops": 6 * values}
    if case["op"] == "project":
        rows, k, n, rank = case["rows"], case["k"], case["n"], case["rank"]
        used = min(case["adapters"], rows)
        bytes_ = rows * k + n * k + 4 * (rows + n) + 2 * rows * n + used * 2 * rank * (k + n) + (4 * rows if used else 0)
        return {"bytes": bytes_, "flops": 2 * rows * (k * n + (rank * (k + n) if used else 0))}
    if case["op"] == "rotate":
        values = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["d"]
        return {"bytes": 4 * values + 4 * case["tokens"] * case["axes"], "flops": 3 * values}
    return {"bytes": 2 * case["copies"] * case["heads"] * (2 * BLOCK * case["d"] + 2 * case["d"] + 8), "flops": 0}


# ---------------------------------------------------------------------------------------- the definition in 64 bits


def _exact_norm(case, state):
    """A few thousand rows at a time: the sum is held in its type, products, units and quotients in 32 bits."""
    outs = []
    for x, r in zip(state["x"].split(4096), state["residual"].split(4096) if case["residual"] else state["x"].split(4096)):
        both = x.double() + r.double() if case["residual"] else x.double()
        h = both.to(x.dtype).double()
        t = (h * state["weight"].double()).float().double()
        unit = (t.abs().max(1, keepdim=True).values / 127.0).float().double()
        q = torch.nan_to_num((t / unit).float().double().round()).clamp(-127, 127)
        over = torch.rsqrt((h * h).mean(1, keepdim=True) + 1e-6)
        outs.append([q * unit * over] + ([both] if case["residual"] else []) + ([t * over] if case["y"] else []))
    return [torch.cat(parts) for parts in zip(*outs)]


def _exact_project(case, state):
    w = state["w"].double() * state["w_scale"].double()[:, None]
    out = (state["x"].double() * state["x_scale"].double()[:, None]) @ w.t().contiguous()
    for a in range(case["adapters"]):
        rows = torch.nonzero(state["adapter_of"] == a)[:, 0]
        if rows.numel():
            x = state["x"][rows].double() * state["x_scale"][rows].double()[:, None]
            inner = x @ state["a"][a].double().t().contiguous()
            out[rows] += float(state["alpha"][a]) * (inner @ state["b"][a].double().t().contiguous())
    return out


def _exact_rotate(case, state):
    axis = [a for a, count in enumerate(_sections(case)) for _ in range(count)]
    pairs = len(axis)
    at = [(2 * i, 2 * i + 1) if case["interleaved"] else (i, i + pairs) for i in range(pairs)]
    first, second = (torch.tensor(c, device="cuda") for c in zip(*at))
    turns = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                        state["positions"].double()[axis].t() * state["freqs"])[:, None]
    outs = []
    for rows in (state["q"], state["k"]):
        x = rows.double()
        z = torch.complex(x[..., first], x[..., second]) * turns
        x[..., first], x[..., second] = z.real, z.imag
        outs.append(x)
    return tuple(outs)


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(case, state)
    if case["op"] == "project":
        return _exact_project(case, state)
    if case["op"] == "rotate":
        return _exact_rotate(case, state)
    scales = []
    for name in ("k_scale", "v_scale"):  # whole pages move as they are: of their parts the scales are computed numbers
        scale = state[name].double()
        scale[state["dst"].long()] = scale[state["src"].long()]
        scales.append(scale)
    return [None, None, scales[0], scales[1], None]
