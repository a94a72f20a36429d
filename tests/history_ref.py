"""Plain 64-bit references of the operators over ordered histories, on the CPU, from their definitions; with bounds of what fp32
arithmetic may add, derived here.

u = 2^-24, half a step of fp32.  A gate s = 1 / (1 + e), 1 - s = e / (1 + e) with e = exp(-|g|) as 2^(-|g| log2 e): the exponent's
product is rounded (|g| u) and so is its factor (|g| u / 2), the power is good to two units; so e is off by (1.5 |g| + 2) u.  The sum
1 + e adds one, its reciprocal two, the product e / (1 + e) one: s and 1 - s are off by at most (1.5 |g| + 7) u of their size.

A state is a sum of products of gates with one value each.  With m = s m + (1 - s) |x| for the sum of their magnitudes, every step
multiplies what is there by a gate (its error, and a rounding) and adds to it (a rounding); splitting a row and joining the parts
multiplies by products of the same gates instead and rounds once or twice more a step: e = s e + ((1.5 |g| + 7) u + 4 u) m.
Gradients go the same way from a row's end.

Below 2^-126 powers of two are 0 and products may be: a gate, a state or a gradient is off by TINY more there, and what it is multiplied
by makes that larger (a gate of exp(-200) times a value of 1e10 is 1e-77 and not 0; a gradient that has faded to 2^-126 is off by
all of it, 2^-126 times a value of 1e10 is 1e-28).  So every step adds TINY times (1 + the magnitudes that it multiplies)."""
import numpy as np

U = 2.0 ** -24
TINY = 2.0 ** -126
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8}  # half a step of a stored number, relative


def gates(g):
    with np.errstate(all="ignore"):
        e = np.exp(-np.abs(g))
        big, small = 1 / (1 + e), e / (1 + e)
    up = g >= 0
    return np.where(up, big, small), np.where(up, small, big), (1.5 * np.minimum(np.abs(g), 120.0) + 7) * U


def by_time(indptr):
    """(t, rows that have an entry number t) for every t."""
    length = np.diff(indptr)
    order = np.argsort(-length, kind="stable")
    n = np.searchsorted(-length[order], -np.arange(length.max() if length.size else 0), side="left")
    return [(t, order[:k]) for t, k in enumerate(n)]


def entries(indptr, ids, V, F):
    """x, s, 1 - s and the gates' errors of every entry; entries without an item keep the state."""
    ids = np.arange(V.shape[0]) if ids is None else np.asarray(ids, dtype=np.int64)
    ok = ((ids >= 0) & (ids < V.shape[0]))[:, None]
    at = np.clip(ids, 0, max(0, V.shape[0] - 1))
    x, g = (V[at], F[at]) if V.shape[0] else (np.zeros((ids.size, V.shape[1])),) * 2
    keep, take, off = gates(g)
    return np.where(ok, x, 0.0), np.where(ok, keep, 1.0), np.where(ok, take, 0.0), np.where(ok, off, 0.0)


def recur(indptr, ids, V, F, H0=None):
    """(last, states, bounds of last's and states' fp32 errors)"""
    indptr = np.asarray(indptr)
    x, keep, take, off = entries(indptr, ids, V, F)
    rows, d = indptr.size - 1, V.shape[1]
    h = np.zeros((rows, d)) if H0 is None else H0.astype(np.float64).copy()
    m, e = np.abs(h), np.zeros((rows, d))
    states, bound = np.zeros_like(x), np.zeros_like(x)
    for t, r in by_time(indptr):
        p = indptr[r] + t
        e[r] += TINY * (1 + m[r] + np.abs(x[p]))
        h[r] = keep[p] * h[r] + take[p] * x[p]
        m[r] = keep[p] * m[r] + take[p] * np.abs(x[p])
        e[r] = keep[p] * e[r] + (off[p] + 4 * U) * m[r]
        states[p], bound[p] = h[r], e[r]
    return h, states, e, bound


def recur_backward(indptr, ids, V, F, states, d_states=None, d_last=None, H0=None):
    """(dV, dF, dH0) and their bounds; states as the kernel was given them."""
    indptr = np.asarray(indptr)
    x, keep, take, off = entries(indptr, ids, V, F)
    rows, d = indptr.size - 1, V.shape[1]
    g = np.zeros((rows, d)) if d_last is None else d_last.astype(np.float64).copy()
    m, e = np.abs(g), np.zeros((rows, d))
    before = np.concatenate([np.zeros((1, d)), states[:-1]]) if states.shape[0] else states
    length = np.diff(indptr)
    first = indptr[:-1][length > 0]
    before[first] = 0.0 if H0 is None else H0[length > 0]
    out = [np.zeros_like(x) for _ in range(4)]
    for t, r in by_time(indptr):
        p = indptr[r + 1] - 1 - t
        if d_states is not None:
            g[r] += d_states[p]
            m[r] += np.abs(d_states[p])
        e[r] += 4 * U * m[r] + TINY * (1 + m[r])
        out[0][p] = take[p] * g[r]
        out[2][p] = take[p] * (e[r] + (off[p] + 2 * U) * m[r]) + TINY * (1 + m[r])
        out[1][p] = g[r] * (before[p] - x[p]) * keep[p] * take[p]
        size = np.abs(before[p]) + np.abs(x[p])
        out[3][p] = keep[p] * take[p] * (np.abs(before[p] - x[p]) * e[r] + (2 * off[p] + 6 * U) * m[r] * size) + 3 * TINY * (1 + m[r]) * (1 + size)
        g[r] *= keep[p]
        m[r] *= keep[p]
        e[r] = keep[p] * e[r] + off[p] * m[r]
    return (out[0], out[1], g), (out[2], out[3], e + U * m)


def sum_rows(indptr, ids, values, E):
    """Sums and bounds: products and sums in any order, a rounding each."""
    indptr, ids = np.asarray(indptr), np.asarray(ids, dtype=np.int64)
    ok = (ids >= 0) & (ids < E.shape[0])
    w = np.where(ok, 1.0 if values is None else np.asarray(values, dtype=np.float64), 0.0)
    X, bound = np.zeros((indptr.size - 1, E.shape[1])), np.zeros((indptr.size - 1, E.shape[1]))
    if E.shape[0] and ids.size:
        with np.errstate(invalid="ignore"):
            part = np.where(ok[:, None], w[:, None] * E[np.clip(ids, 0, E.shape[0] - 1)], 0.0)
        owner = np.repeat(np.arange(indptr.size - 1), np.diff(indptr))
        inside = slice(indptr[0], indptr[-1])
        np.add.at(X, owner, part[inside])
        np.add.at(bound, owner, np.abs(part[inside]))
    return X, bound * (np.diff(indptr)[:, None] + 1) * U


def beam(ids, scores, lse, totals, beams, temperature=1.0, last=None, end=-1, lengths=None, factors=None):
    """Every step one IEEE operation in fp32, as defined."""
    f = np.float32
    rows, k = ids.shape
    out = [], [], [], []
    with np.errstate(all="ignore"):
        for g in range(0, rows, beams):
            cand = []
            for r in range(g, g + beams):
                before = f(0.0 if r == g else -np.inf) if totals is None else totals[r]
                over = last is not None and last[r] == end
                length = (0 if lengths is None else int(lengths[r])) + (0 if over else 1)
                for j in range(k):
                    if over:
                        total, item = (before if j == 0 else f(-np.inf)), end
                    else:
                        item = int(ids[r, j])
                        total = f(before + f(f(scores[r, j] / f(temperature)) - (f(0) if lse is None else lse[r]))) if item >= 0 else f(-np.inf)
                    key = total if factors is None else f(total * factors[min(max(length, 0), len(factors) - 1)])
                    if key > -np.inf:
                        cand.append((-float(key), r, j, item, total, length))
            cand.sort(key=lambda c: c[:3])
            cand = cand[:beams] + [(0, -1, 0, -1, f(-np.inf), 0)] * (beams - len(cand))
            for o, i in zip(out, (1, 3, 4, 5)):
                o.extend(c[i] for c in cand)
    return np.array(out[0]), np.array(out[1]), np.array(out[2], dtype=f), np.array(out[3])
