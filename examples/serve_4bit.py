"""Train a small model, cut its item table to 4 bits an entry and answer from it.

    python examples/serve_4bit.py [--nodes 30000] [--d 64] [--group 32] [--epochs 4]

Rows of a synthetic link matrix are held out, embedded from three quarters of their links (als_solve_rows) and answered
twice: from the fp32 table (als_topk) and from the 4-bit one (als_scores, als_select).  The rules of the second answer: links
that a row was folded in from are not returned again (a set of allowed items per row), popular items are held back a little
(a bias per item).  Printed: bytes of both tables, Recall@20 of both answers on the held-out links, and one row's items with their
probabilities among all items.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2112_02194_amd import binding as als  # noqa: E402
from synth import holdout_split, make_problem, transpose_csr  # noqa: E402


def allowed_sets(indptr, indices, rows, items):
    """One bit per row and item, clear for the row's links, as the int32 words that als.Rules takes."""
    bits = torch.ones((rows, (items + 31) // 32 * 32), dtype=torch.bool, device=indices.device)
    owner = torch.repeat_interleave(torch.arange(rows, device=indices.device), indptr[1:] - indptr[:-1])
    bits[owner, indices.long()] = False
    weight = 1 << torch.arange(32, device=indices.device)
    words = (bits.view(rows, -1, 32) * weight).sum(2)  # 0 .. 2^32 - 1
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


def recall(ids, indptr, indices, k):
    """Share of each row's held-out links among its first k answers, over the rows that have any."""
    total, rows = 0.0, 0
    for q in range(ids.shape[0]):
        held = set(indices[indptr[q]:indptr[q + 1]].tolist())
        if held:
            total += len(held.intersection(ids[q, :k].tolist())) / min(k, len(held))
            rows += 1
    return total / rows


def main(nodes=30000, d=64, group=32, epochs=4, k=20, temperature=1.0, device=0):
    dev = torch.device("cuda", device)
    ctx = als.Context(device)
    p = make_problem("c3", rows=nodes, cols=nodes, d=d)
    split = holdout_split(p.indptr, p.indices, seed=99)
    n_train, n_test, n = split["train_rows"].numel(), split["test_rows"].numel(), p.cols
    tr_ptr, tr_idx = split["train"]
    tt_ptr, tt_idx, _ = transpose_csr(n_train, n, tr_ptr, tr_idx)
    Y, Yt = als.Csr(n_train, n, tr_ptr.to(dev), tr_idx.to(dev)), als.Csr(n, n_train, tt_ptr.to(dev), tt_idx.to(dev))
    W, H = p.W0[split["train_rows"]].to(dev), p.H0.to(dev)
    params = als.make_params(p.alpha, p.lam)
    for _ in range(epochs):
        als.als_epoch(ctx, Y, Yt, W, H, params)

    # rows that were not trained, from the links that are given
    given = als.Csr(n_test, n, *(t.to(dev) for t in split["given"]))
    X = torch.zeros((n_test, d), device=dev)
    als.als_solve_rows(ctx, given, H, als.als_gramian(ctx, H), params, X)

    full_ids, _ = als.als_topk(ctx, X, H, k, given)

    T = als.als_quantize(ctx, H, group)
    popularity = (tt_ptr[1:] - tt_ptr[:-1]).to(dev)
    rules = als.Rules(bias=-1e-3 * torch.log1p(popularity.float()), allowed=allowed_sets(given.indptr, given.indices, n_test, n))
    scores = als.als_scores(ctx, X, T)
    ids, best, lse = als.als_select(ctx, scores, k, rules, temperature)
    probability = torch.exp(best / temperature - lse[:, None])
    als.als_status_sync(ctx)

    held = [t.numpy() for t in split["held"]]
    result = {"bytes": (H.numel() * 4, T.codes.numel() + 2 * T.scales.numel()),
              "recall": (recall(full_ids.cpu(), *held, k), recall(ids.cpu(), *held, k)),
              "ids": ids.cpu(), "probability": probability.cpu(), "given": split["given"]}
    ctx.close()
    return result


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--nodes", type=int, default=30000)
    ap.add_argument("--d", type=int, default=64)
    ap.add_argument("--group", type=int, default=32)
    ap.add_argument("--epochs", type=int, default=4)
    r = main(**vars(ap.parse_args()))
    print("item table: %.1f MB in fp32, %.1f MB in 4 bits" % tuple(b / 1e6 for b in r["bytes"]))
    print("Recall@20: %.4f from fp32, %.4f from 4 bits" % r["recall"])
    print("first row:", ", ".join("%d (%.2e)" % (i, p) for i, p in zip(r["ids"][0, :5].tolist(), r["probability"][0, :5].tolist())))
