"""The operators of ordered histories, as cases that can be timed and compared: a query from a history whose order counts, its
gradients, and answers of several items one after the other.

Six kinds of call, each through the public entry points of ``paper_2112_02194_amd.binding``:

``recur``  a gated linear recurrence over the rows of a sparse matrix, entries in their stored order:
           h = s h + (1 - s) V[item] with s = sigmoid(F[item]) for every entry of a row; the last state of each row, or all states
``back``   its gradients, one row of both per entry, and those of the first states
``step``   one more entry for every row, from the states of parent rows
``sum``    sums of a table's rows over the rows of a sparse matrix (table gradients from those of the entries; sums over histories)
``clip``   the norm over many tensors, and all of them scaled where it is above a bound
``beam``   the best continuations of groups of beams from each beam's best items, and the beams' states in the new order

Each has a plain form in elementary torch operations, in 32 bits and rounded once at the end (``own`` is false), and a
definition in 64 bits (``exact``).  Inputs are drawn on the GPU from the seed.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
END = 0  # the item that ends a beam
_context = None


def context():
    """A program keeps one context for its whole life."""
    global _context
    if _context is None:
        from paper_2112_02194_amd import binding

        _context = binding.Context(0)
    return _context


# --------------------------------------------------------------------------- the cases

def _recur(kind, rows, mean, longest, items, d, dtype, out, states, first):
    """mean, longest: of the rows' lengths, which are all the same where the two are equal; items: rows of the tables, 0 for
    tables with a row for each entry; out: type of states and gradients; states: all of them, or each row's last one; first:
    rows begin at given states."""
    return {"kind": kind, "rows": rows, "mean": mean, "longest": longest, "items": items, "d": d, "dtype": dtype, "out": out,
            "states": states, "first": first}


def _step(groups, beams, items, d, dtype):
    return {"kind": "step", "groups": groups, "beams": beams, "items": items, "d": d, "dtype": dtype}


def _sum(rows, entries, d, dtype, out, by_item, weights):
    """by_item: each entry of the table belongs to one row (an item), a few rows have many; otherwise rows are short lists over
    the table."""
    return {"kind": "sum", "rows": rows, "entries": entries, "d": d, "dtype": dtype, "out": out, "by_item": by_item, "weights": weights}


def _clip(tensors, values, dtype, factor):
    """factor: the bound over the norm that is expected."""
    return {"kind": "clip", "tensors": tensors, "values": values, "dtype": dtype, "factor": factor}


def _beam(groups, beams, k, items, d, steps, ended):
    """steps: items that a beam's sequence has room for; ended: some beams have come to their end, and lengths count."""
    return {"kind": "beam", "groups": groups, "beams": beams, "k": k, "items": items, "d": d, "steps": steps, "ended": ended}


def listed():
    return [
        # one page of beams takes its next items: launches count
        {"name": "step_page", **_step(64, 8, 30_000, 64, "f32")},
        # one page of visitors with short histories
        {"name": "recur_page", **_recur("recur", 64, 30, 400, 30_000, 64, "f32", "f32", False, False)},
        # queries for all rows of a training matrix: lengths spread widely, popular items often
        {"name": "recur_rows", **_recur("recur", 300_000, 20, 20_000, 1_000_003, 128, "bf16", "f32", False, False)},
        # training on a few long sequences, all states, tables with a row for each entry
        {"name": "recur_long", **_recur("recur", 16, 65_537, 65_537, 0, 128, "f32", "f32", True, True)},
        # gradients of a training matrix' rows
        {"name": "back_rows", **_recur("back", 100_000, 20, 20_000, 300_007, 64, "f32", "f32", True, False)},
        # gradients of a few long sequences of bf16 tables
        {"name": "back_long", **_recur("back", 16, 65_537, 65_537, 0, 128, "bf16", "f32", True, True)},
        # weighted sums over one page of histories
        {"name": "sum_page", **_sum(4096, 100_003, 64, "bf16", "f32", False, True)},
        # an item table's gradient from those of all entries: items with one entry and with tens of thousands
        {"name": "sum_items", **_sum(1_000_003, 6_000_000, 64, "f32", "f32", True, False)},
        # the parameters of a small model: many tensors, odd sizes, both types
        {"name": "clip_many", **_clip(60, 2_000_000, "both", 0.1)},
        # gradients of two large tables
        {"name": "clip_tables", **_clip(2, 1_000_000_000, "f32", 0.5)},
        # one visitor who waits
        {"name": "beam_one", **_beam(1, 8, 8, 30_000, 64, 50, False)},
        # a block of sessions at once, each beam with a set of allowed items of its own
        {"name": "beam_block", **_beam(128, 32, 32, 1_000_000, 128, 200, True)},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["recur", "recur", "recur", "back", "back", "step", "sum", "sum", "clip", "beam"])
    d = rng.choice([16, 32, 64, 64, 128, 128])
    dtype, out = rng.choice(["f32", "f32", "bf16"]), rng.choice(["f32", "f32", "bf16"])
    if kind in ("recur", "back"):
        entries = _log_int(rng, 200, (400_000_000 if kind == "recur" else 130_000_000) // d)
        longest = _log_int(rng, 1, min(entries, 65_537))
        mean = longest if rng.random() < 0.3 else _log_int(rng, 1, min(longest, 60))
        rows = max(1, entries // mean)
        return _recur(kind, rows, mean, longest, rng.choice([0, _log_int(rng, 1000, 1_000_003)]), d, dtype, out,
                      kind == "back" or rng.random() < 0.5, rng.random() < 0.5)
    if kind == "step":
        beams = rng.choice([1, 4, 8, 32, 64])
        return _step(_log_int(rng, 1, 1_000_000 // beams), beams, _log_int(rng, 1000, 1_000_003), d, dtype)
    if kind == "sum":
        entries, by_item = _log_int(rng, 1000, 400_000_000 // d), rng.random() < 0.6
        rows = _log_int(rng, 1, min(entries, 1_000_003 if by_item else 20_000_000 // d))
        return _sum(rows, entries, d, dtype, out, by_item, rng.random() < 0.5)
    if kind == "clip":
        tensors = rng.choice([1, 2, _log_int(rng, 1, 60), _log_int(rng, 1, 60)])
        return _clip(tensors, _log_int(rng, 1000 * tensors, 1_000_000_000), rng.choice(["f32", "bf16", "both"]), rng.choice([0.02, 0.5, 2.0]))
    beams = rng.choice([1, 2, 4, 5, 8, 16, 32, 50, 64])
    items = _log_int(rng, 1000, 1_000_000)
    return _beam(_log_int(rng, 1, max(1, min(4096, 4_000_000_000 // (beams * items)))), beams, rng.choice([beams, 64]), items, d,
                 rng.choice([10, 50, 200]), rng.random() < 0.5)


# --------------------------------------------------------------------------- inputs

def _table(rows, d, gen):
    """Rows as training leaves them: a decaying spectrum in a rotated basis and norms that differ from row to row."""
    scale = 0.3 / math.sqrt(d) * torch.arange(1, d + 1, device=DEV, dtype=torch.float32) ** -0.5
    basis, _ = torch.linalg.qr(torch.randn((d, d), device=DEV, generator=gen))
    x = torch.randn((rows, d), device=DEV, generator=gen) @ (scale[:, None] * basis)
    return x.mul_(torch.exp(0.5 * torch.randn((rows, 1), device=DEV, generator=gen)))


def _popular(n, items, gen):
    """Item ids, a few of them often."""
    rank = torch.rand(n, device=DEV, generator=gen, dtype=torch.float64) ** 3
    return ((rank * items).to(torch.int64) * 2654435761) % items


def _lengths(case, gen):
    """Row lengths: a few long rows, many short ones, some of them empty."""
    rows, mean, longest = case["rows"], case["mean"], case["longest"]
    if mean == longest:
        return torch.full((rows,), mean, dtype=torch.int64, device=DEV)
    # the same lengths for every seed, in another order
    rank = torch.arange(rows, dtype=torch.float64, device=DEV)
    length = (mean / 2.7 * (1.0 - (rank + 0.5) / rows) ** (-2.0 / 3.0) + 0.5).to(torch.int64).clamp_(1, longest)
    if rows > 1:
        length[::10] = 0
    return length[torch.randperm(rows, device=DEV, generator=gen)]


def _pointers(length):
    indptr = torch.zeros(length.numel() + 1, dtype=torch.int64, device=DEV)
    torch.cumsum(length, 0, out=indptr[1:])
    return indptr


def _prepare_recur(case, gen, state):
    d, dtype, out = case["d"], DTYPES[case["dtype"]], DTYPES[case["out"]]
    length = _lengths(case, gen)
    indptr = state["indptr"] = _pointers(length)
    nnz = int(indptr[-1])
    state["longest"] = max(1, int(length.max()))
    items = case["items"] or nnz
    state["ids"] = _popular(nnz, items, gen).to(torch.int32) if case["items"] else None
    state["V"] = _table(items, d, gen).to(dtype)
    # gates from a few entries of memory to some hundreds
    state["F"] = (1.5 + 1.5 * torch.randn((items, d), device=DEV, generator=gen)).to(dtype)
    state["first"] = _table(case["rows"], d, gen).to(out) if case["first"] else None
    if case["kind"] == "back":
        state["h"] = _plain_recur(state)[1].to(out)
        state["d_states"] = torch.randn((nnz, d), device=DEV, generator=gen).mul_(0.01).to(out)
        state["d_last"] = torch.randn((case["rows"], d), device=DEV, generator=gen).mul_(0.01).to(out)


def _prepare_beam(case, gen, state):
    rows, k, items = case["groups"] * case["beams"], case["k"], case["items"]
    # each beam's best items as a selection leaves them: best first, with the log of the sum over all items
    top = 5.0 + torch.randn((rows, 1), device=DEV, generator=gen) * 0.3
    state["scores"] = top - torch.cumsum(torch.rand((rows, k), device=DEV, generator=gen) * 0.2, 1)
    start = _popular(rows, items, gen)[:, None] + torch.randint(1, max(2, items // k), (rows, 1), device=DEV, generator=gen) * torch.arange(k, device=DEV)
    state["ids"] = (start % items).to(torch.int32)
    state["lse"] = math.log(items) + 0.5 + torch.randn(rows, device=DEV, generator=gen) * 0.2
    state["totals"] = -8.0 + torch.randn(rows, device=DEV, generator=gen)
    state["items"] = _popular(rows, items, gen).to(torch.int32).clamp_(min=END + 1)
    state["lengths"] = torch.full((rows,), case["steps"] // 2, dtype=torch.int32, device=DEV)
    state["factors"] = None
    if case["ended"]:
        over = torch.rand(rows, device=DEV, generator=gen) < 0.15
        state["items"][over] = END
        state["lengths"][over] -= torch.randint(1, 4, (rows,), device=DEV, generator=gen, dtype=torch.int32)[over]
        state["factors"] = ((5.0 + torch.arange(case["steps"] + 1, device=DEV, dtype=torch.float64)) / 6.0).pow(-0.6).float()
    # what goes with a beam: its query, its items so far, the set of items that it may still take
    word = lambda n: torch.randint(-2 ** 31, 2 ** 31, (rows, n), device=DEV, generator=gen, dtype=torch.int64).to(torch.int32)  # noqa: E731
    state["states"] = [_table(rows, case["d"], gen), word(case["steps"]).bitwise_and_(0xFFFFF), word((items + 31) // 32)]
    state["out"] = [torch.empty_like(t) for t in state["states"]]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1_000_003 * seed + 31)
    state = {"case": dict(case)}
    kind = case["kind"]
    if kind in ("recur", "back"):
        _prepare_recur(case, gen, state)
    elif kind == "step":
        rows, dtype = case["groups"] * case["beams"], DTYPES[case["dtype"]]
        state["V"] = _table(case["items"], case["d"], gen).to(dtype)
        state["F"] = (1.5 + 1.5 * torch.randn((case["items"], case["d"]), device=DEV, generator=gen)).to(dtype)
        state["H"] = _table(rows, case["d"], gen)
        state["items"] = _popular(rows, case["items"], gen).to(torch.int32)
        row = torch.arange(rows, device=DEV)
        state["parents"] = (row - row % case["beams"] + torch.randint(0, case["beams"], (rows,), device=DEV, generator=gen)).to(torch.int32)
    elif kind == "sum":
        rows, n, d = case["rows"], case["entries"], case["d"]
        if case["by_item"]:
            owner = _popular(n, rows, gen)
            state["ids"] = torch.argsort(owner, stable=True).to(torch.int32)
            state["indptr"] = _pointers(torch.bincount(owner, minlength=rows))
            state["E"] = torch.randn((n, d), device=DEV, generator=gen).mul_(0.01).to(DTYPES[case["dtype"]])
        else:  # lists of about 20
            rows_of = torch.randint(0, 41, (rows,), device=DEV, generator=gen)
            state["indptr"] = _pointers(rows_of)
            state["ids"] = _popular(int(state["indptr"][-1]), n, gen).to(torch.int32)
            state["E"] = _table(n, d, gen).to(DTYPES[case["dtype"]])
        nnz = state["ids"].numel()
        state["weights"] = 0.5 + torch.rand(nnz, device=DEV, generator=gen) if case["weights"] else None
    elif kind == "clip":
        share = [(0.618034 * n) % 1.0 + 1e-3 for n in range(1, case["tensors"] + 1)]
        total = sum(v * v for v in share)
        sizes = [max(1, int(v * v / total * case["values"])) for v in share]
        state["tensors"] = []
        for n, size in enumerate(sizes):
            x = torch.randn(size, device=DEV, generator=gen).mul_(0.01)
            state["tensors"].append(x.to(torch.bfloat16) if case["dtype"] == "bf16" or (case["dtype"] == "both" and n % 2) else x)
        state["bound"] = case["factor"] * 0.01 * math.sqrt(sum(sizes))
        state["out"] = [torch.empty_like(x) for x in state["tensors"]]
    else:
        _prepare_beam(case, gen, state)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    return state


# --------------------------------------------------------------------------- the plain forms

def _owner(indptr, n):
    """Row of each entry."""
    return torch.repeat_interleave(torch.arange(indptr.numel() - 1, device=DEV), indptr[1:] - indptr[:-1], output_size=n)


def _plain_scan(a, b, longest):
    """h[t] = a[t] h[t-1] + b[t] along the first axis, where a is 0 at each row's first entry: by doubling."""
    reach = 1
    while reach < longest:  # every value stands for `reach` entries up to its own
        more = a[reach:] * b[:-reach]
        b = torch.cat((b[:reach], b[reach:] + more))
        a = torch.cat((a[:reach], a[reach:] * a[:-reach]))
        reach *= 2
    return b


def _plain_entries(state):
    V, F = (t if state["ids"] is None else t[state["ids"].long()] for t in (state["V"], state["F"]))
    V, F = V.float(), F.float()
    return V, torch.sigmoid(F), torch.sigmoid(-F)


def _plain_recur(state):
    """(last state of each row, all states)"""
    indptr = state["indptr"]
    x, keep, take = _plain_entries(state)
    b = take * x
    some = indptr[1:] > indptr[:-1]
    starts = indptr[:-1][some]
    first = torch.zeros((indptr.numel() - 1, x.shape[1]), device=DEV) if state["first"] is None else state["first"].float()
    b[starts] += keep[starts] * first[some]
    keep[starts] = 0.0
    h = _plain_scan(keep, b, state["longest"])
    last = first.clone()
    last[some] = h[indptr[1:][some] - 1]
    return last, h


def _plain_back(state):
    indptr = state["indptr"]
    x, keep, take = _plain_entries(state)
    some = indptr[1:] > indptr[:-1]
    starts, ends = indptr[:-1][some], indptr[1:][some] - 1
    first = torch.zeros((indptr.numel() - 1, x.shape[1]), device=DEV) if state["first"] is None else state["first"].float()
    before = state["h"].float().roll(1, 0)
    before[starts] = first[some]
    b = state["d_states"].float().index_add(0, ends, state["d_last"].float()[some])
    a = keep.roll(-1, 0)  # of the next entry
    a[ends] = 0.0
    delta = _plain_scan(a.flip(0), b.flip(0), state["longest"]).flip(0)
    d_first = state["d_last"].float().clone()
    d_first[some] = (keep * delta)[starts]
    return take * delta, delta * (before - x) * keep * take, d_first


def _plain_beam(state):
    case = state["case"]
    groups, beams, k = case["groups"], case["beams"], case["k"]
    row = torch.arange(groups * beams, device=DEV)
    over = state["items"] == END if case["ended"] else torch.zeros_like(row, dtype=torch.bool)
    temperature = torch.full((1,), TEMPERATURE, device=DEV)
    total = state["totals"][:, None] + (state["scores"] / temperature - state["lse"][:, None])
    place = torch.arange(k, device=DEV)
    total = torch.where(over[:, None], torch.where(place == 0, state["totals"][:, None], -math.inf), total)
    items = torch.where(over[:, None], torch.full_like(state["ids"], END), state["ids"])
    lengths = state["lengths"] + (~over).int()
    key = total if state["factors"] is None else total * state["factors"][lengths.long()][:, None]
    # one whole number orders by key first and by ascending place among equal keys
    bits = (key.reshape(groups, -1) + 0.0).view(torch.int32)
    bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
    order = (bits.long() << 32) | (0x7FFFFFFF - torch.arange(beams * k, device=DEV))
    best = torch.topk(order, beams, 1).indices + beams * k * torch.arange(groups, device=DEV)[:, None]
    best = best.reshape(-1)
    parents = torch.div(best, k, rounding_mode="floor")
    answer = {"parents": parents.int(), "items": items.reshape(-1)[best], "totals": total.reshape(-1)[best], "lengths": lengths[parents]}
    return answer, [t[parents] for t in state["states"]]


TEMPERATURE = 0.9


def _plain(state):
    case = state["case"]
    kind = case["kind"]
    if kind == "recur":
        out = DTYPES[case["out"]]
        last, h = _plain_recur(state)
        return {"last": last.to(out), "states": h.to(out)} if case["states"] else {"last": last.to(out)}
    if kind == "back":
        dV, dF, d_first = _plain_back(state)
        out = DTYPES[case["out"]]
        got = {"dV": dV.to(out), "dF": dF.to(out)}
        return {**got, "d_first": d_first.to(out)} if case["first"] else got
    if kind == "step":
        items = state["items"].long()
        V, F = state["V"][items].float(), state["F"][items].float()
        return torch.sigmoid(F) * state["H"][state["parents"].long()] + torch.sigmoid(-F) * V
    if kind == "sum":
        E = state["E"][state["ids"].long()].float()
        if state["weights"] is not None:
            E *= state["weights"][:, None]
        X = torch.zeros((case["rows"], case["d"]), device=DEV)
        return X.index_add_(0, _owner(state["indptr"], E.shape[0]), E).to(DTYPES[case["out"]])
    if kind == "clip":
        tensors = state["tensors"]
        norm = torch.sqrt(torch.stack([x.double().square().sum() for x in tensors]).sum())
        factor = (state["bound"] / norm).clamp(max=1.0).float()
        return {"norm": norm, "tensors": [(x.float() * factor).to(x.dtype) for x in tensors]}
    answer, states = _plain_beam(state)
    return {**answer, "states": states}


# --------------------------------------------------------------------------- one pass

def run(state):
    if not own:
        return _plain(state)
    from paper_2112_02194_amd import binding as als

    case, ctx = state["case"], context()
    kind = case["kind"]
    if kind in ("recur", "back"):
        out = DTYPES[case["out"]]
        Y = als.Csr(case["rows"], state["V"].shape[0], state["indptr"], state["ids"])
        if kind == "recur":
            last, states = als.als_recur(ctx, Y, state["V"], state["F"], H0=state["first"], all_states=case["states"], dtype=out)
            return {"last": last, "states": states} if case["states"] else {"last": last}
        dV, dF, d_first = als.als_recur_backward(ctx, Y, state["V"], state["F"], state["h"], d_states=state["d_states"],
                                                 d_last=state["d_last"], H0=state["first"], dtype=out)
        return {"dV": dV, "dF": dF, "d_first": d_first} if case["first"] else {"dV": dV, "dF": dF}
    if kind == "step":
        return als.als_recur_step(ctx, state["items"], state["V"], state["F"], state["H"], parents=state["parents"])
    if kind == "sum":
        Y = als.Csr(case["rows"], state["E"].shape[0], state["indptr"], state["ids"], state["weights"])
        return als.als_sum_rows(ctx, Y, state["E"], dtype=DTYPES[case["out"]])
    if kind == "clip":
        norm = als.als_clip(ctx, state["tensors"], state["bound"], out=state["out"])
        return {"norm": norm, "tensors": state["out"]}
    parents, items, totals, lengths = als.als_beam(ctx, state["ids"], state["scores"], state["lse"], state["totals"], case["beams"],
                                                   temperature=TEMPERATURE, last=state["items"] if case["ended"] else None, end=END,
                                                   lengths=state["lengths"], factors=state["factors"])
    states = als.als_reorder(ctx, parents, case["beams"], state["states"], out=state["out"])
    return {"parents": parents, "items": items, "totals": totals, "lengths": lengths, "states": states}


# --------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    kind = case["kind"]
    if kind in ("recur", "back"):
        rows, d, e, o = case["rows"], case["d"], BYTES[case["dtype"]], BYTES[case["out"]]
        nnz = int(rows * case["mean"])  # the mean of the lengths
        items = min(case["items"] or nnz, nnz)
        read = 2 * items * d * e + 8 * rows + (4 * nnz if case["items"] else 0) + (rows * d * o if case["first"] else 0)
        if kind == "recur":
            return {"bytes": read + rows * d * o + (nnz * d * o if case["states"] else 0), "flops": 12 * nnz * d}
        return {"bytes": read + 4 * nnz * d * o + rows * d * o * (2 if case["first"] else 1), "flops": 20 * nnz * d}
    if kind == "step":
        rows, d, e = case["groups"] * case["beams"], case["d"], BYTES[case["dtype"]]
        return {"bytes": 2 * min(rows, case["items"]) * d * e + 8 * rows + 8 * rows * d, "flops": 12 * rows * d}
    if kind == "sum":
        rows, n, d = case["rows"], case["entries"], case["d"]
        nnz = n if case["by_item"] else 20 * rows
        read = min(n, nnz) * d * BYTES[case["dtype"]] + 8 * rows + nnz * (8 if case["weights"] else 4)
        return {"bytes": read + rows * d * BYTES[case["out"]], "flops": (2 if case["weights"] else 1) * nnz * d}
    if kind == "clip":
        each = {"f32": 4, "bf16": 2, "both": 3}[case["dtype"]]
        return {"bytes": 2 * each * case["values"], "flops": 3 * case["values"]}
    rows = case["groups"] * case["beams"]
    row = 4 * (case["d"] + case["steps"] + (case["items"] + 31) // 32)
    return {"bytes": rows * (8 * case["k"] + 12 + 16 + 2 * row), "flops": 4 * rows * case["k"]}


# --------------------------------------------------------------------------- the definitions in 64 bits

def _one_after_the_other(state, case, step):
    """Calls step(entries, rows, time) for the first entries of all rows that have one, then their second ones, and so on."""
    indptr = state["indptr"]
    length = indptr[1:] - indptr[:-1]
    order = torch.argsort(length, descending=True, stable=True)
    sorted_length = length[order].cpu()
    # rows that have an entry number t, for each t
    counts = (sorted_length.numel() - torch.searchsorted(sorted_length.flip(0).contiguous(), torch.arange(1, int(sorted_length[0]) + 1))).tolist()
    for t, n in enumerate(counts):
        step(order[:n], t)


def _exact_recur(state, case):
    start, ids = state["indptr"][:-1], state["ids"]
    nnz, d = int(state["indptr"][-1]), case["d"]
    last = torch.zeros((case["rows"], d), dtype=torch.float64, device=DEV) if state["first"] is None else state["first"].double()
    states = torch.empty((nnz, d), dtype=torch.float64, device=DEV) if case["states"] else None

    def step(rows, t):
        entry = start[rows] + t
        item = entry if ids is None else ids[entry].long()
        keep = 1.0 / (1.0 + torch.exp(-state["F"][item].double()))
        x = state["V"][item].double()
        h = x + keep * (last[rows] - x)
        last[rows] = h
        if states is not None:
            states[entry] = h

    _one_after_the_other(state, case, step)
    return {"last": last, "states": states} if case["states"] else {"last": last}


def _exact_back(state, case):
    end, ids = state["indptr"][1:] - 1, state["ids"]
    start = state["indptr"][:-1]
    delta = state["d_last"].double()
    dV, dF = (torch.empty(state["h"].shape, dtype=torch.float64, device=DEV) for _ in range(2))
    first = torch.zeros_like(delta) if state["first"] is None else state["first"].double()

    def step(rows, t):
        entry = end[rows] - t
        item = entry if ids is None else ids[entry].long()
        keep = 1.0 / (1.0 + torch.exp(-state["F"][item].double()))
        now = delta[rows] + state["d_states"][entry].double()
        before = torch.where((entry == start[rows])[:, None], first[rows], state["h"][(entry - 1).clamp(min=0)].double())
        dV[entry] = now - keep * now
        dF[entry] = now * (before - state["V"][item].double()) * (keep - keep * keep)
        delta[rows] = keep * now

    _one_after_the_other(state, case, step)
    return {"dV": dV, "dF": dF, "d_first": delta} if case["first"] else {"dV": dV, "dF": dF}


def _exact_beam(state, case):
    """Totals by 64-bit sums, taken at the places that order by 32-bit sums as they are defined."""
    groups, beams, k = case["groups"], case["beams"], case["k"]
    shape = (groups, beams, k)
    over = (state["items"] == END).view(groups, beams, 1) if case["ended"] else torch.zeros((groups, beams, 1), dtype=torch.bool, device=DEV)
    live = state["scores"].double() / float(torch.tensor(TEMPERATURE, dtype=torch.float32)) - state["lse"].double()[:, None]
    total = state["totals"].double().view(groups, beams, 1) + torch.where(over, 0.0, live.view(shape))
    total = total.masked_fill(over & (torch.arange(k, device=DEV) > 0), -math.inf)
    key = total
    if case["ended"]:
        length = state["lengths"].view(groups, beams, 1) + (~over).int()
        key = total * state["factors"].double()[length.long()]
    best = torch.argsort(key.view(groups, -1), dim=1, descending=True, stable=True)[:, :beams]
    # what is copied has no other value; near a tie in 32 bits 64 may order otherwise
    return {"parents": None, "items": None, "totals": total.view(groups, -1).gather(1, best).view(-1), "lengths": None, "states": [None] * 3}


def exact(case, seed):
    state = prepare(case, seed)
    kind = case["kind"]
    if kind == "recur":
        return _exact_recur(state, case)
    if kind == "back":
        return _exact_back(state, case)
    if kind == "step":
        items = state["items"].long()
        keep = 1.0 / (1.0 + torch.exp(-state["F"][items].double()))
        x = state["V"][items].double()
        return x + keep * (state["H"].double()[state["parents"].long()] - x)
    if kind == "sum":  # a running sum along all entries would lose digits: rows in blocks of their own
        indptr, ids, E = state["indptr"], state["ids"].long(), state["E"]
        X = torch.zeros((case["rows"], case["d"]), dtype=torch.float64, device=DEV)
        owner = torch.bucketize(torch.arange(ids.numel(), device=DEV), indptr[1:], right=True)
        for c in range(0, case["d"], 16):
            part = E[:, c:c + 16].double()[ids]
            if state["weights"] is not None:
                part *= state["weights"].double()[:, None]
            X[:, c:c + 16] = torch.zeros((case["rows"], 16), dtype=torch.float64, device=DEV).scatter_add_(0, owner[:, None].expand(-1, 16), part)
        return X
    if kind == "clip":
        total = 0.0
        for x in state["tensors"]:
            for part in x.split(1 << 26):
                total = total + torch.linalg.vector_norm(part.double()) ** 2
        norm = torch.sqrt(total)
        factor = min(1.0, state["bound"] / float(norm))
        return {"norm": norm, "tensors": [x.double() * factor for x in state["tensors"]]}
    return _exact_beam(state, case)
