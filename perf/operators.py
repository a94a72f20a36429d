"""The operators that answer from a trained table, as cases that can be timed and compared.

Four kinds of call, each through the public entry points of ``paper_2112_02194_amd.binding``:

``quantize``  an embedding table is cut to 4 bits an entry with one scale per group of entries, and read back
``scores``    inner products of queries with all items of a 4-bit table
``adjust``    scores changed by rules: penalties for items a row has had before, biases, sets of allowed items
``select``    the best items of (changed) scores and the log of the sum of their exponentials

Each has a plain form in elementary torch operations, in 32 bits and rounded once at the end (``own`` is false), and a
definition in 64 bits (``exact``).  Inputs are drawn on the GPU from the seed.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_context = None


def context():
    """A program keeps one context for its whole life."""
    global _context
    if _context is None:
        from paper_2112_02194_amd import binding

        _context = binding.Context(0)
    return _context


# --------------------------------------------------------------------------- the cases

def _quantize(items, d, dtype, group):
    return {"kind": "quantize", "items": items, "d": d, "dtype": dtype, "group": group}


def _scores(queries, items, d, dtype, group, out):
    return {"kind": "scores", "queries": queries, "items": items, "d": d, "dtype": dtype, "group": group, "out": out}


def _rows(kind, queries, items, dtype, history, bias, entries, allowed, penalties):
    """history, entries: mean length of a row's list (0: none); bias: one value an item; allowed: none, shared (one set
    for all rows) or rows (a set each); penalties: shared, or rows (three numbers each)."""
    return {"kind": kind, "queries": queries, "items": items, "dtype": dtype, "history": history, "bias": bias,
            "entries": entries, "allowed": allowed, "penalties": penalties}


def listed():
    return [
        # a small catalogue: launches count
        {"name": "quantize_small", **_quantize(1500, 16, "f32", 16)},
        # a bf16 table of odd length, the coarsest groups that its rows have
        {"name": "quantize_bf16", **_quantize(1_000_003, 64, "bf16", 64)},
        # the headline's item table, 5 GB
        {"name": "quantize_large", **_quantize(10_000_000, 128, "f32", 32)},
        # one user who waits, 1M items
        {"name": "scores_one", **_scores(1, 1_000_003, 128, "f32", 32, "f32")},
        # one user against a table that is large even at 4 bits
        {"name": "scores_one_large", **_scores(1, 20_000_000, 128, "bf16", 32, "f32")},
        # one page of users against a small catalogue
        {"name": "scores_page", **_scores(64, 30_000, 64, "f32", 64, "f32")},
        # evaluation: a block of rows against 1M items, bf16 scores
        {"name": "scores_block", **_scores(512, 1_000_000, 64, "bf16", 32, "bf16")},
        # one user with a long history, every rule
        {"name": "adjust_one", **_rows("adjust", 1, 30_000, "f32", 2000, True, 64, "rows", "rows")},
        # a block of rows, one set of items on sale for all
        {"name": "adjust_block", **_rows("adjust", 256, 1_000_000, "f32", 30, True, 0, "shared", "shared")},
        # one user who waits, items had before leave the answer or sink
        {"name": "select_one", **_rows("select", 1, 1_000_003, "f32", 200, False, 0, "none", "shared"), "k": 50, "temperature": 0.7},
        # one page of users, every rule
        {"name": "select_page", **_rows("select", 64, 30_000, "f32", 60, True, 16, "rows", "rows"), "k": 20, "temperature": 1.0},
        # evaluation: a block of bf16 rows, Recall@50
        {"name": "select_block", **_rows("select", 512, 1_000_000, "bf16", 15, False, 0, "none", "shared"), "k": 50, "temperature": 1.0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quantize", "scores", "scores", "scores", "adjust", "adjust", "select", "select", "select"])
    d = rng.choice([16, 32, 64, 64, 128, 128])
    group = rng.choice([g for g in (16, 32, 64, 128) if g <= d])
    dtype = rng.choice(["f32", "f32", "bf16"])
    if kind == "quantize":
        return _quantize(_log_int(rng, 1000, 10_000_000), d, dtype, group)
    if kind == "scores":
        queries = rng.choice([1, 1, 2, 3, _log_int(rng, 1, 512), _log_int(rng, 1, 512)])
        return _scores(queries, _log_int(rng, 1000, min(20_000_000, 256_000_000 // queries)), d, dtype, group,
                       rng.choice(["f32", "bf16"]))
    queries = rng.choice([1, 2, _log_int(rng, 1, 512), _log_int(rng, 1, 512)])
    items = _log_int(rng, 1000, min(20_000_000, 256_000_000 // queries))
    case = _rows(kind, queries, items, dtype, rng.choice([0, 15, 60, _log_int(rng, 10, 4000)]), rng.random() < 0.5,
                 rng.choice([0, 16]), rng.choice(["none", "shared", "rows"]), rng.choice(["shared", "rows"]))
    if kind == "select":
        case.update(k=rng.choice([1, 10, 20, 50, 64]), temperature=rng.choice([0.5, 1.0, 1.7]))
    return case


# --------------------------------------------------------------------------- inputs

def _table(rows, d, gen):
    """Rows as training leaves them: a decaying spectrum in a rotated basis and norms that differ from row to row."""
    scale = 0.3 / math.sqrt(d) * torch.arange(1, d + 1, device=DEV, dtype=torch.float32) ** -0.5
    basis, _ = torch.linalg.qr(torch.randn((d, d), device=DEV, generator=gen))
    x = torch.randn((rows, d), device=DEV, generator=gen) @ (scale[:, None] * basis)
    return x.mul_(torch.exp(0.5 * torch.randn((rows, 1), device=DEV, generator=gen)))


def _packed(case, gen):
    """A 4-bit table: codes from -7 to 7 as the rounding of normal entries leaves them, two a byte, the even one in the
    low half, in two's complement; one bf16 scale per group, spread like the rows' norms."""
    n, d, g = case["items"], case["d"], case["group"]
    byte = torch.arange(256, device=DEV)
    weight = torch.exp(-0.5 * ((torch.arange(16, device=DEV) - 16 * (torch.arange(16, device=DEV) > 7)) / 3.0) ** 2)
    weight[8] = 0.0  # -8 is not used
    chance = (weight[byte & 15] * weight[byte >> 4]).double()
    edges = torch.cumsum(chance / chance.sum(), 0).float()
    codes = torch.empty((n, d // 2), dtype=torch.uint8, device=DEV)
    for r0 in range(0, n, 1 << 20):
        u = torch.rand((min(1 << 20, n - r0), d // 2), device=DEV, generator=gen)
        codes[r0:r0 + u.shape[0]] = torch.searchsorted(edges, u).clamp_(max=255).to(torch.uint8)
    scales = 0.03 / math.sqrt(d) * torch.exp(0.5 * torch.randn((n, d // g), device=DEV, generator=gen))
    codes = torch.where((codes & 15) == 8, codes ^ 8, codes)  # the last edge is rounded: keep to the codes in use
    return torch.where((codes >> 4) == 8, codes ^ 128, codes), scales.to(torch.bfloat16)


def _lists(queries, items, mean, gen, distinct):
    """Lists of item ids, a few popular ones often: row lengths from none to several times the mean."""
    length = (mean * -torch.log(1.0 - torch.rand(queries, device=DEV, generator=gen))).to(torch.int64)
    if queries == 1:
        length[0] = mean
    owner = torch.repeat_interleave(torch.arange(queries, device=DEV), length)
    rank = torch.rand(owner.numel(), device=DEV, generator=gen, dtype=torch.float64) ** 3
    ids = ((rank * items).to(torch.int64) * 2654435761) % items
    if distinct:
        key = torch.unique(owner * items + ids)
        owner = torch.div(key, items, rounding_mode="floor")
        ids = key - owner * items
    indptr = torch.zeros(queries + 1, dtype=torch.int64, device=DEV)
    torch.cumsum(torch.bincount(owner, minlength=queries), 0, out=indptr[1:])
    return indptr, ids.to(torch.int32)


def _allowed(rows, items, gen):
    """One bit an item, set for about three quarters of them; with several rows one of them allows nothing."""
    words = (items + 31) // 32
    a = torch.randint(-2 ** 31, 2 ** 31, (rows, words), device=DEV, generator=gen, dtype=torch.int64)
    b = torch.randint(-2 ** 31, 2 ** 31, (rows, words), device=DEV, generator=gen, dtype=torch.int64)
    bits = (a | b).to(torch.int32)
    if rows > 1:
        bits[rows // 2] = 0
    return bits


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1_000_003 * seed + 29)
    state = {"case": dict(case)}
    dtype = DTYPES[case["dtype"]]
    if case["kind"] == "quantize":
        state["X"] = _table(case["items"], case["d"], gen).to(dtype)
    elif case["kind"] == "scores":
        state["codes"], state["scales"] = _packed(case, gen)
        state["Q"] = _table(case["queries"], case["d"], gen).to(dtype)
    else:
        nq, n = case["queries"], case["items"]
        S = torch.empty((nq, n), dtype=dtype, device=DEV)
        for q in range(nq):  # a row at a time: no second matrix in 32 bits
            S[q] = torch.randn(n, device=DEV, generator=gen) * 1.5
        state["S"] = S
        state["history"] = _lists(nq, n, case["history"], gen, False) if case["history"] else None
        state["bias"] = 0.5 * torch.randn(n, device=DEV, generator=gen) if case["bias"] else None
        state["entries"] = None
        if case["entries"]:
            indptr, ids = _lists(nq, n, case["entries"], gen, True)
            state["entries"] = (indptr, ids, 2.0 * torch.randn(ids.numel(), device=DEV, generator=gen))
        state["allowed"] = None if case["allowed"] == "none" else _allowed(nq if case["allowed"] == "rows" else 1, n, gen)
        # repetition, presence, frequency
        state["penalties"] = None
        if case["penalties"] == "rows":
            low, span = torch.tensor([1.0, 0.0, 0.0], device=DEV), torch.tensor([0.5, 0.8, 0.3], device=DEV)
            state["penalties"] = low + span * torch.rand((nq, 3), device=DEV, generator=gen)
        if case["kind"] == "adjust":
            state["out"] = torch.empty_like(S)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    return state


SHARED_PENALTIES = (1.3, 0.4, 0.1)


# --------------------------------------------------------------------------- the plain forms

def _plain_quantized(X, group):
    n, d = X.shape
    x = X.float().view(n, d // group, group)
    # a tensor as the divisor: a true division, not a product with the reciprocal
    scale = (x.abs().amax(2, keepdim=True) / torch.full((1,), 7.0, device=X.device)).to(torch.bfloat16).float()
    code = (x / scale).round().clamp(-7.0, 7.0)
    return (torch.where(scale > 0, code, torch.zeros_like(code)) * scale).view(n, d)


def _plain_values(codes, scales, d, group):
    half = torch.stack((codes & 15, codes >> 4), 2).view(codes.shape[0], d // group, group)
    value = half.float()
    value -= 16.0 * (half > 7)
    value *= scales.float()[:, :, None]
    return value.view(-1, d)


def _plain_dense(lists, values, shape):
    indptr, ids = lists[0], lists[1].long()
    owner = torch.repeat_interleave(torch.arange(shape[0], device=DEV), indptr[1:] - indptr[:-1])
    dense = torch.zeros(shape[0] * shape[1], device=DEV)
    return dense.index_add_(0, owner * shape[1] + ids, values).view(shape)


def _plain_adjusted(state):
    x = state["S"].float()
    if state["history"] is not None:
        p = state["penalties"]
        if p is None:
            p = torch.tensor([SHARED_PENALTIES], device=DEV)
        r, presence, frequency = p[:, 0:1], p[:, 1:2], p[:, 2:3]
        count = _plain_dense(state["history"], torch.ones(state["history"][1].numel(), device=DEV), x.shape)
        x = torch.where(count > 0, torch.where(x > 0, x / r, x * r) - frequency * count - presence, x)
    if state["bias"] is not None:
        x = x + state["bias"]
    if state["entries"] is not None:
        x = x + _plain_dense(state["entries"], state["entries"][2], x.shape)
    if state["allowed"] is not None:
        bits = (state["allowed"][:, :, None] >> torch.arange(32, device=DEV, dtype=torch.int32)) & 1
        x = torch.where(bits.view(bits.shape[0], -1)[:, :x.shape[1]] == 1, x, torch.full((1,), -math.inf, device=DEV))
    return x


def _plain_selected(x, k, temperature):
    nq, n = x.shape
    t = x / torch.full((1,), temperature, device=DEV)
    top = t.amax(1, keepdim=True)
    lse = torch.where(top > -math.inf, top + torch.log(torch.exp(t - top).sum(1, keepdim=True)), top)
    # one whole number orders by score first and by ascending id among equal scores
    bits = (x + 0.0).view(torch.int32)
    bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
    key = (bits.long() << 32) | (0x7FFFFFFF - torch.arange(n, device=DEV))
    ids = torch.topk(key, min(k, n), 1).indices
    scores = torch.gather(x, 1, ids)
    ids = torch.where(scores > -math.inf, ids, torch.full_like(ids, -1)).to(torch.int32)
    out_ids = torch.full((nq, k), -1, dtype=torch.int32, device=DEV)
    out_scores = torch.full((nq, k), -math.inf, device=DEV)
    out_ids[:, :ids.shape[1]], out_scores[:, :ids.shape[1]] = ids, scores
    return {"ids": out_ids, "scores": out_scores, "lse": lse[:, 0]}


def _plain(state):
    case = state["case"]
    if case["kind"] == "quantize":
        return _plain_quantized(state["X"], case["group"])
    if case["kind"] == "scores":
        values = _plain_values(state["codes"], state["scales"], case["d"], case["group"])
        return (state["Q"].float() @ values.T).to(DTYPES[case["out"]])
    x = _plain_adjusted(state)
    if case["kind"] == "adjust":
        return x.to(DTYPES[case["dtype"]])
    return _plain_selected(x, case["k"], case["temperature"])


# --------------------------------------------------------------------------- one pass

def run(state):
    if not own:
        return _plain(state)
    from paper_2112_02194_amd import binding as als

    case, ctx = state["case"], context()
    if case["kind"] == "quantize":
        return als.als_dequantize(ctx, als.als_quantize(ctx, state["X"], case["group"]))
    if case["kind"] == "scores":
        return als.als_scores(ctx, state["Q"], als.QTable(state["codes"], state["scales"]), dtype=DTYPES[case["out"]])
    shape = (case["queries"], case["items"])
    repetition, presence, frequency = SHARED_PENALTIES
    rules = als.Rules(history=None if state["history"] is None else als.Csr(*shape, *state["history"]),
                      repetition=repetition, presence=presence, frequency=frequency, penalties=state["penalties"],
                      bias=state["bias"], entries=None if state["entries"] is None else als.Csr(*shape, *state["entries"]),
                      allowed=state["allowed"])
    if case["kind"] == "adjust":
        return als.als_adjust(ctx, state["S"], rules, out=state["out"])
    ids, scores, lse = als.als_select(ctx, state["S"], case["k"], rules, case["temperature"])
    return {"ids": ids, "scores": scores, "lse": lse}


# --------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    n, es = case["items"], 4 if case["dtype"] == "f32" else 2
    if case["kind"] in ("quantize", "scores"):
        d = case["d"]
        packed = n * (d // 2 + 2 * (d // case["group"]))
        if case["kind"] == "quantize":  # the table read, the packed one written and read, 32 bits an entry written
            return {"bytes": n * d * (es + 4) + 2 * packed, "flops": 4 * n * d}
        nq = case["queries"]
        return {"bytes": packed + nq * d * es + nq * n * (4 if case["out"] == "f32" else 2), "flops": 2 * nq * n * d}
    nq = case["queries"]
    lists = nq * (4 * case["history"] + 8 * case["entries"]) + (16 * (nq + 1) if case["history"] or case["entries"] else 0)
    sets = (n + 31) // 32 * 4 * {"none": 0, "shared": 1, "rows": nq}[case["allowed"]]
    read = nq * n * es + lists + sets + (4 * n if case["bias"] else 0)
    if case["kind"] == "adjust":
        return {"bytes": read + nq * n * es, "flops": 2 * nq * n}
    return {"bytes": read + nq * (8 * case["k"] + 4), "flops": 4 * nq * n}


# --------------------------------------------------------------------------- the definitions in 64 bits

def _exact_row(state, q):
    """Row q after the rules, entry by entry of its lists."""
    x = state["S"][q].double()
    if state["history"] is not None:
        p = SHARED_PENALTIES if state["penalties"] is None else state["penalties"][q].tolist()
        p = [float(torch.tensor(v, dtype=torch.float32)) for v in p]
        indptr, ids = state["history"]
        had, times = torch.unique(ids[int(indptr[q]):int(indptr[q + 1])].long(), return_counts=True)
        v = x[had]
        x[had] = torch.maximum(v, torch.zeros_like(v)) / p[0] + torch.minimum(v, torch.zeros_like(v)) * p[0] - times * p[2] - p[1]
    if state["bias"] is not None:
        x += state["bias"].double()
    if state["entries"] is not None:
        indptr, ids, values = state["entries"]
        a, b = int(indptr[q]), int(indptr[q + 1])
        x[ids[a:b].long()] += values[a:b].double()
    if state["allowed"] is not None:
        words = state["allowed"][q if state["allowed"].shape[0] > 1 else 0].long()
        item = torch.arange(x.numel(), device=x.device)
        x.masked_fill_(((words[item // 32] >> (item % 32)) & 1) == 0, -math.inf)
    return x


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "quantize":
        out = torch.empty((case["items"], case["d"]), dtype=torch.float64, device=DEV)
        for r0 in range(0, case["items"], 1 << 20):
            for c0 in range(0, case["d"], case["group"]):
                x = state["X"][r0:r0 + (1 << 20), c0:c0 + case["group"]].double()
                s = (x.abs().max(1).values / 7.0).to(torch.bfloat16).double()[:, None]
                out[r0:r0 + (1 << 20), c0:c0 + case["group"]] = torch.nan_to_num(x / s).round().clamp(-7, 7) * s
        return out
    if case["kind"] == "scores":
        nq, n, d, g = case["queries"], case["items"], case["d"], case["group"]
        out = torch.empty((nq, n), dtype=torch.float64, device=DEV)
        Qt = state["Q"].double().T.contiguous()
        for r0 in range(0, n, 1 << 20):
            byte = state["codes"][r0:r0 + (1 << 20)].to(torch.int16)
            v = torch.empty((byte.shape[0], d), dtype=torch.float64, device=DEV)
            v[:, 0::2] = ((byte & 15) ^ 8).double() - 8.0
            v[:, 1::2] = ((byte >> 4) ^ 8).double() - 8.0
            total = 0.0
            for c in range(d // g):
                total = total + state["scales"][r0:r0 + (1 << 20), c:c + 1].double() * (v[:, c * g:(c + 1) * g] @ Qt[c * g:(c + 1) * g])
            out[:, r0:r0 + (1 << 20)] = total.T
        return out
    rows = range(case["queries"])
    if case["kind"] == "adjust":
        return torch.stack([_exact_row(state, q) for q in rows])
    scores = torch.full((case["queries"], case["k"]), -math.inf, dtype=torch.float64, device=DEV)
    lse = torch.empty(case["queries"], dtype=torch.float64, device=DEV)
    temperature = float(torch.tensor(case["temperature"], dtype=torch.float32))
    for q in rows:
        x = _exact_row(state, q)
        best = torch.topk(x, min(case["k"], x.numel())).values
        scores[q, :best.numel()] = best
        lse[q] = torch.logsumexp(x / temperature, 0)
    return {"ids": None, "scores": scores, "lse": lse}
