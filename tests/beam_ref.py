"""What als_beam answers, from the definition of a candidate alone: every candidate is written down with its total first, those that are
none are taken out, and only then is anything ordered."""
import numpy as np


def candidates(ids, scores, lse, totals, first, beams, temperature, last, end, lengths):
    """(row, place, item, total, length) of a group's candidates."""
    f = np.float32
    out = []
    for row in range(first, first + beams):
        so_far = f(0) if totals is None else totals[row]
        if totals is None and row != first:
            continue
        length = 0 if lengths is None else int(lengths[row])
        if last is not None and last[row] == end:
            some = [(0, end, so_far, length)]
        else:
            less = f(0) if lse is None else lse[row]
            some = [(j, int(ids[row, j]), f(so_far + f(f(scores[row, j] / f(temperature)) - less)), length + 1)
                    for j in range(ids.shape[1]) if ids[row, j] >= 0]
        out.extend((row, j, item, total, many) for j, item, total, many in some if not (np.isnan(total) or total == -np.inf))
    return out


def beam(ids, scores, lse, totals, beams, temperature=1.0, last=None, end=-1, lengths=None, factors=None):
    """(parents, items, totals, lengths), every step one IEEE operation in fp32."""
    f = np.float32
    answer = []
    with np.errstate(all="ignore"):
        for first in range(0, ids.shape[0], beams):
            ordered = []
            for row, j, item, total, length in candidates(ids, scores, lse, totals, first, beams, temperature, last, end, lengths):
                key = total if factors is None else f(total * factors[min(length, len(factors) - 1)])
                if key > -np.inf:  # neither -inf nor NaN
                    ordered.append((-float(key), row, j, item, total, length))
            ordered.sort(key=lambda c: c[:3])
            answer += [(row, item, total, length) for _, row, _, item, total, length in ordered[:beams]]
            answer += [(-1, -1, f(-np.inf), 0)] * max(0, beams - len(ordered))
    rows = list(zip(*answer))
    return np.array(rows[0]), np.array(rows[1]), np.array(rows[2], dtype=f), np.array(rows[3])
