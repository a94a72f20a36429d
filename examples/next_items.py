"""Learn how long a history's items count, and continue histories by several items.

    python examples/next_items.py [--nodes 20000] [--d 64] [--epochs 3] [--steps 5]

An item table is trained by alternating least squares (als_epoch).  A row's stored entries are then taken as a history in its order:
als_recur turns it into a query, h = s h + (1 - s) V[item] with a gate s per item and column.  The gates' table is learned by
gradient steps: after every entry the query should be near the next entry's item.  als_recur gives all queries,
als_recur_backward the gradients of every entry, als_sum_rows those of each item, als_clip bounds them.  Held-out rows
are continued by beam search: als_scores against the 4-bit table, als_select, als_beam, als_reorder, als_recur_step.
Printed: the loss and the gradients' norm at each step, and one row's best continuations with their log-probabilities.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2112_02194_amd import binding as als  # noqa: E402
from synth import holdout_split, make_problem, transpose_csr  # noqa: E402


def entries_by_item(ids, items):
    """For every item the entries that store it, as a Csr over entries."""
    counts = torch.bincount(ids.long(), minlength=items)
    indptr = torch.zeros(items + 1, dtype=torch.int64, device=ids.device)
    torch.cumsum(counts, 0, out=indptr[1:])
    return als.Csr(items, ids.numel(), indptr, torch.argsort(ids, stable=True).to(torch.int32))


def next_entries(indptr, n):
    """For every entry the one behind it in its row, and whether there is one."""
    last = torch.zeros(n, dtype=torch.bool, device=indptr.device)
    last[(indptr[1:] - 1)[indptr[1:] > indptr[:-1]]] = True
    return torch.arange(1, n + 1, device=indptr.device).clamp_(max=n - 1), ~last


def loss_and_gradients(ctx, Y, by_item, V, F):
    """Mean of |query after an entry - next entry's item|^2 / 2, and its gradients with respect to the tables as the recurrence reads
    them (the items that the queries are compared with are held)."""
    _, states = als.als_recur(ctx, Y, V, F, all_states=True)
    behind, some = next_entries(Y.indptr, Y.nnz)
    off = torch.where(some[:, None], states - V[Y.indices[behind].long()], 0.0)
    count = some.sum()
    dV, dF, _ = als.als_recur_backward(ctx, Y, V, F, states, d_states=off / count)
    return off.square().sum() / (2 * count), als.als_sum_rows(ctx, by_item, dV), als.als_sum_rows(ctx, by_item, dF)


def continue_histories(ctx, Y, V, F, T, beams, steps, k, temperature):
    """The best `beams` continuations of every row by `steps` items: items [rows, beams, steps] and log-probabilities [rows, beams]."""
    rows = Y.rows * beams
    H = als.als_recur(ctx, Y, V, F)[0].repeat_interleave(beams, 0)
    taken = torch.full((rows, steps), -1, dtype=torch.int32, device=V.device)
    every = torch.arange(0, rows * steps + 1, steps, device=V.device)
    totals = None
    for t in range(steps):
        scores = als.als_scores(ctx, H, T)
        rules = als.Rules(history=als.Csr(rows, V.shape[0], every, taken.view(-1)), presence=1e9)  # no item twice (-1 is none)
        ids, best, lse = als.als_select(ctx, scores, k, rules, temperature)
        parents, items, totals, _ = als.als_beam(ctx, ids, best, lse, totals, beams, temperature)
        als.als_reorder(ctx, parents, beams, [taken])
        taken[:, t] = items
        H = als.als_recur_step(ctx, items, V, F, H, parents)
    return taken.view(Y.rows, beams, steps), totals.view(Y.rows, beams)


def main(nodes=20000, d=64, epochs=3, gate_steps=8, rate=1000.0, bound=5e-4, beams=4, steps=5, temperature=0.1, answered=64, device=0):
    dev = torch.device("cuda", device)
    ctx = als.Context(device)
    p = make_problem("c3", rows=nodes, cols=nodes, d=d)
    split = holdout_split(p.indptr, p.indices, seed=99)
    n_train, n = split["train_rows"].numel(), p.cols
    tr_ptr, tr_idx = split["train"]
    tt_ptr, tt_idx, _ = transpose_csr(n_train, n, tr_ptr, tr_idx)
    Y, Yt = als.Csr(n_train, n, tr_ptr.to(dev), tr_idx.to(dev)), als.Csr(n, n_train, tt_ptr.to(dev), tt_idx.to(dev))
    W, V = p.W0[split["train_rows"]].to(dev), p.H0.to(dev)
    params = als.make_params(p.alpha, p.lam)
    for _ in range(epochs):
        als.als_epoch(ctx, Y, Yt, W, V, params)

    F = torch.full_like(V, 1.0)
    by_item, history = entries_by_item(Y.indices, n), []
    for _ in range(gate_steps):
        loss, _, dF = loss_and_gradients(ctx, Y, by_item, V, F)
        norm = als.als_clip(ctx, [dF], bound)
        F.sub_(dF, alpha=rate)
        history.append((float(loss), float(norm)))

    ptr, ids = split["given"]
    given = als.Csr(answered, n, ptr[:answered + 1].to(dev), ids[:int(ptr[answered])].to(dev))
    items, totals = continue_histories(ctx, given, V, F, als.als_quantize(ctx, V), beams, steps, beams, temperature)
    als.als_status_sync(ctx)
    result = {"training": history, "items": items.cpu(), "log_probability": totals.cpu(), "gates": torch.sigmoid(F).mean().item()}
    ctx.close()
    return result


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--nodes", type=int, default=20000)
    ap.add_argument("--d", type=int, default=64)
    ap.add_argument("--epochs", type=int, default=3)
    ap.add_argument("--steps", type=int, default=5)
    r = main(**vars(ap.parse_args()))
    for step, (loss, norm) in enumerate(r["training"]):
        print("gates, step %d: loss %.6f, norm of the gradients %.3e" % (step, loss, norm))
    for beam in range(r["items"].shape[1]):
        print("first row:", ", ".join("%d" % i for i in r["items"][0, beam].tolist()), "(%.3f)" % r["log_probability"][0, beam])
