"""Plain 64-bit references of the operators that answer from trained tables, on the CPU, from their definitions."""
import numpy as np
import torch


def bf16(x):
    """fp32 -> bf16 (nearest even) -> fp32, as numpy."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).float().numpy()


def quantize(x, group):
    """(codes int, scales) of an fp32 table; every step is one IEEE operation in fp32, as defined."""
    n, d = x.shape
    g = x.astype(np.float32).reshape(n, d // group, group)
    with np.errstate(all="ignore"):
        top = np.abs(g).max(axis=2)  # NaN stays
        scale = bf16(top / np.float32(7.0))
        code = np.rint(g / scale[:, :, None])
        code = np.where((scale > 0) & np.isfinite(scale), 1.0, np.nan)[:, :, None] * np.clip(code, -7, 7)
    return np.nan_to_num(code, nan=0.0).astype(np.int64).reshape(n, d), scale


def pack(code):
    u = (code & 15).astype(np.uint8)
    return u[:, 0::2] | (u[:, 1::2] << 4)


def values(code, scale):
    n, d = code.shape
    with np.errstate(all="ignore"):
        return code * np.repeat(scale.astype(np.float64), d // scale.shape[1], axis=1)


def adjust(x, history=None, repetition=1.0, presence=0.0, frequency=0.0, penalties=None, bias=None, entries=None, allowed=None):
    """Rules on fp64 scores; lists are (indptr, ids[, values]) as numpy.  Returns the scores and, for a bound of the rounding,
    the sum of the magnitudes that went into each."""
    x = x.astype(np.float64).copy()
    mag = np.abs(x)
    rows, cols = x.shape
    with np.errstate(all="ignore"):
        for q in range(rows):
            r, p, f = (repetition, presence, frequency) if penalties is None else penalties[q].astype(np.float64)
            if history is not None:
                ids = history[1][history[0][q]:history[0][q + 1]]
                ids, c = np.unique(ids[(ids >= 0) & (ids < cols)], return_counts=True)
                v = x[q, ids]
                v = np.where(v > 0, v / r, v * r)
                mag[q, ids] = np.abs(v) + np.abs(f * c) + abs(p)
                x[q, ids] = v - f * c - p
            if bias is not None:
                x[q] += bias.astype(np.float64)
                mag[q] += np.abs(bias)
            if entries is not None:
                last = {}
                for i in range(entries[0][q], entries[0][q + 1]):
                    if 0 <= entries[1][i] < cols:
                        last[int(entries[1][i])] = 1.0 if entries[2] is None else float(entries[2][i])
                for i, v in last.items():
                    x[q, i] += v
                    mag[q, i] += abs(v)
            if allowed is not None:
                words = allowed[q if allowed.shape[0] > 1 else 0].astype(np.int64) & 0xFFFFFFFF
                i = np.arange(cols)
                x[q, ((words[i // 32] >> (i % 32)) & 1) == 0] = -np.inf
    return x, mag


def select(x, k, temperature=1.0):
    """Best k of every row: descending, equal scores by ascending id, no -inf and no NaN; log-sum-exp over the row."""
    rows, cols = x.shape
    ids = np.full((rows, k), -1, dtype=np.int64)
    scores = np.full((rows, k), -np.inf)
    lse = np.full(rows, -np.inf)
    for q in range(rows):
        ok = np.flatnonzero(x[q] > -np.inf)
        order = ok[np.argsort(-x[q, ok], kind="stable")][:k]
        ids[q, :order.size], scores[q, :order.size] = order, x[q, order]
        if np.isnan(x[q]).any():
            lse[q] = np.nan
        elif ok.size:
            m = x[q, ok].max()
            lse[q] = m if np.isinf(m) else m / temperature + np.log(np.exp((x[q, ok] - m) / temperature).sum())
    return ids, scores, lse
