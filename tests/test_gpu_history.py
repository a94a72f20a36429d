"""Ordered histories on the GPU: the gated recurrence with its gradients and its step, sums over lists, clipping, beams.

References are plain 64-bit computations on the CPU (history_ref, which derives the bounds of the fp32 arithmetic beside them); a
result stored in bf16 adds half a step of it.  What is moved or chosen has to be equal to the bit."""
import numpy as np
import pytest
import torch

import history_ref as ref
from gpu_util import f64, say
from paper_2112_02194_amd import binding as als

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ctx(gpu_device):
    c = als.Context(0)
    yield c
    c.close()


def stored(bound, want, dtype):
    """The bound with the rounding to the type it is stored in (and what fp32 keeps below its normal range)."""
    half = ref.HALF[str(dtype).split(".")[1]]
    return bound * (1 + half) + half * np.abs(want) + 1e-37


def near(got, want, bound, dtype):
    got = f64(got)
    assert got.shape == want.shape
    off = np.abs(got - want) / stored(bound, want, dtype)
    worst = float(off.max()) if off.size else 0.0
    assert worst <= 1.0


def padded(rows, d, dtype, dev, pad=0, fill=float("nan")):
    """Rows further apart than they are long, between others that must stay as they are."""
    big = torch.full((rows + 2, d + pad), fill, dtype=dtype, device=dev)
    return big, big[1:rows + 1, :d]


def put(t, dev, pad=0):
    if not pad:
        return t.to(dev)
    _, inner = padded(t.shape[0], t.shape[1], t.dtype, dev, pad)
    inner.copy_(t.to(dev))
    return inner


def tables(n, d, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    V = torch.randn((n, d), generator=gen)
    F = 1.5 + 2.0 * torch.randn((n, d), generator=gen)
    if n > 8:
        F[3] = 30.0   # keeps for ever
        F[4] = -30.0  # forgets at once
        F[5, ::2] = 200.0
        V[6] *= 1e10
    return V.to(dtype), F.to(dtype)


SHORT = [0, 1, 2, 3, 0, 7, 8, 9, 15, 16, 17, 31, 33, 0, 0, 63, 64, 65, 100, 1, 1, 1, 127, 128, 129, 200, 0]
LONG = [1, 255, 0, 256, 257, 511, 513, 700, 1023, 1025, 0, 1500, 2]


def history(lengths, items, seed, stray=True):
    gen = torch.Generator().manual_seed(seed)
    ptr = torch.zeros(len(lengths) + 1, dtype=torch.int64)
    ptr[1:] = torch.cumsum(torch.tensor(lengths, dtype=torch.int64), 0)
    n = int(ptr[-1])
    ids = (torch.rand(n, generator=gen) ** 2 * items).to(torch.int32)
    if stray and n > 20:
        ids[torch.randint(0, n, (n // 10,), generator=gen)] = -1  # padding
        ids[n // 2] = items
        ids[0] = -7
        ids[n - 1] = 2 ** 31 - 1
    return ptr, ids


def csr(ptr, ids, cols, dev, values=None):
    return als.Csr(ptr.numel() - 1, cols, ptr.to(dev), None if ids is None else ids.to(dev), None if values is None else values.to(dev))


# ------------------------------------------------------------------------------------------------ the recurrence

@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF16, F32), (F32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("lengths", [SHORT, LONG, [1], [0], [5000, 3]], ids=["short", "long", "one", "none", "5000"])
def test_recur_matches_the_definition(ctx, gpu_device, d, dtype, out, lengths):
    items = 50
    V, F = tables(items, d, dtype, d)
    ptr, ids = history(lengths, items, len(lengths))
    for first, pad in ((True, 0), (False, 16)):
        say(f"als_recur d={d} {dtype} -> {out}, {len(lengths)} rows of up to {max(lengths)}, first={first} pad={pad}")
        H0 = torch.randn((len(lengths), d), generator=torch.Generator().manual_seed(9)).to(out) if first else None
        want, want_states, bound, bound_states = ref.recur(ptr.numpy(), ids.numpy(), f64(V), f64(F), None if H0 is None else f64(H0))
        big, last = padded(len(lengths), d, out, gpu_device, pad, 7.0)
        big_states, states = padded(ids.numel(), d, out, gpu_device, pad, 7.0)
        Y = csr(ptr, ids, items, gpu_device)
        tv, tf, th = put(V, gpu_device, pad), put(F, gpu_device, pad), None if H0 is None else put(H0, gpu_device, pad)
        als.als_recur(ctx, Y, tv, tf, th, last=last, states=states)
        alone, none = als.als_recur(ctx, Y, tv, tf, th, dtype=out)
        torch.cuda.synchronize()
        assert none is None
        near(last, want, bound, out)
        near(alone, want, bound, out)
        near(states, want_states, bound_states, out)
        last.fill_(7.0)
        states.fill_(7.0)
        assert torch.all(big == 7.0) and torch.all(big_states == 7.0)


@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF16, F32), (F32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("lengths", [SHORT, LONG, [1], [0], [5000, 3]], ids=["short", "long", "one", "none", "5000"])
def test_recur_backward_matches_the_formula(ctx, gpu_device, d, dtype, out, lengths):
    items, rows = 50, len(lengths)
    V, F = tables(items, d, dtype, d + 1)
    ptr, ids = history(lengths, items, rows + 1)
    gen = torch.Generator().manual_seed(5)
    n = ids.numel()
    for which, pad in (("all", 0), ("states", 16), ("last", 8)):
        say(f"als_recur_backward d={d} {dtype}, {out}, {rows} rows of up to {max(lengths)}, gradients of {which} pad={pad}")
        H0 = torch.randn((rows, d), generator=gen).to(out) if which != "last" else None
        states = torch.from_numpy(ref.recur(ptr.numpy(), ids.numpy(), f64(V), f64(F), None if H0 is None else f64(H0))[1]).to(out)
        ds = torch.randn((n, d), generator=gen).to(out) if which != "last" else None
        dl = torch.randn((rows, d), generator=gen).to(BF16 if which == "all" else F32) if which != "states" else None
        want, bound = ref.recur_backward(ptr.numpy(), ids.numpy(), f64(V), f64(F), f64(states), None if ds is None else f64(ds),
                                         None if dl is None else f64(dl), None if H0 is None else f64(H0))
        types = (out, out, F32)
        got = [padded(k, d, t, gpu_device, pad, 7.0) for k, t in zip((n, n, rows), types)]
        dev = [None if t is None else put(t, gpu_device, pad) for t in (V, F, states, ds, dl, H0)]
        als.als_recur_backward(ctx, csr(ptr, ids, items, gpu_device), *dev, out=[t for _, t in got])
        torch.cuda.synchronize()
        for (big, t), w, b, kind in zip(got, want, bound, types):
            near(t, w, b, kind)
            t.fill_(7.0)
            assert torch.all(big == 7.0)


@pytest.mark.parametrize("d,dtype", [(16, F32), (128, F32), (64, BF16), (32, BF16)])
def test_entries_that_take_their_own_rows(ctx, gpu_device, d, dtype):
    lengths = LONG + SHORT
    say(f"als_recur, als_recur_backward without ids, d={d} {dtype}")
    n = sum(lengths)
    V, F = tables(n, d, dtype, 2)
    ptr, _ = history(lengths, 1, 0)
    Y = csr(ptr, None, n, gpu_device)
    want, want_states, bound, bound_states = ref.recur(ptr.numpy(), None, f64(V), f64(F))
    last, states = als.als_recur(ctx, Y, V.to(gpu_device), F.to(gpu_device), all_states=True)
    torch.cuda.synchronize()
    near(last, want, bound, F32)
    near(states, want_states, bound_states, F32)
    ds = torch.randn((n, d), generator=torch.Generator().manual_seed(5))
    want, bound = ref.recur_backward(ptr.numpy(), None, f64(V), f64(F), f64(states), f64(ds))
    dV, dF, dH0 = als.als_recur_backward(ctx, Y, V.to(gpu_device), F.to(gpu_device), states, d_states=ds.to(gpu_device))
    torch.cuda.synchronize()
    near(dV, want[0], bound[0], F32)
    near(dF, want[1], bound[1], F32)
    assert dH0 is None


def test_gradients_are_differences(ctx, gpu_device):
    """Against differences of the 64-bit reference along random directions.  The kernels' own error is bounded as everywhere; the
    difference's, with a step of 1e-5 and third derivatives of some tens of the values, is below 1e-8 of the sum of magnitudes."""
    say("als_recur, als_recur_backward, als_sum_rows: directional differences")
    d, items = 16, 12
    lengths = [0, 5, 130, 1, 64, 300]
    rng = np.random.default_rng(1)
    V, F, H0 = (torch.from_numpy(rng.normal(size=s)).float() for s in ((items, d), (items, d), (len(lengths), d)))
    ptr, ids = history(lengths, items, 4)
    n = ids.numel()
    ws, wl = torch.from_numpy(rng.normal(size=(n, d))).float(), torch.from_numpy(rng.normal(size=(len(lengths), d))).float()
    Y = csr(ptr, ids, items, gpu_device)
    dev = [t.to(gpu_device) for t in (V, F)]
    _, states = als.als_recur(ctx, Y, *dev, H0.to(gpu_device), all_states=True)
    dV, dF, dH0 = als.als_recur_backward(ctx, Y, *dev, states, ws.to(gpu_device), wl.to(gpu_device), H0.to(gpu_device))
    ok = (ids >= 0) & (ids < items)
    order = torch.argsort(torch.where(ok, ids, items), stable=True).to(torch.int32)
    heads = torch.zeros(items + 1, dtype=torch.int64)
    heads[1:] = torch.cumsum(torch.bincount(ids[ok].long(), minlength=items), 0)
    T = csr(heads, order[:int(ok.sum())], n, gpu_device)
    gV, gF = (als.als_sum_rows(ctx, T, t) for t in (dV, dF))
    torch.cuda.synchronize()

    def loss(V, F, H0):
        last, states, _, _ = ref.recur(ptr.numpy(), ids.numpy(), V, F, H0)
        return (f64(ws) * states).sum() + (f64(wl) * last).sum()

    args = [f64(t) for t in (V, F, H0)]
    for k, grad in enumerate((gV, gF, dH0)):
        for _ in range(3):
            way = rng.normal(size=args[k].shape)
            up, down = (loss(*[a + (s * 1e-5 * way if j == k else 0) for j, a in enumerate(args)]) for s in (1, -1))
            size = np.abs(f64(grad) * way).sum()
            # gradients are off by about 100 roundings (gates of |g| < 5, memory of some tens of entries) of sums whose magnitudes
            # are at most tens of times their values
            assert abs((up - down) / 2e-5 - (f64(grad) * way).sum()) <= 3000 * ref.U * size


@pytest.mark.parametrize("d,dtype,out", [(16, F32, F32), (32, BF16, F32), (64, F32, BF16), (128, BF16, BF16), (128, F32, F32)])
def test_long_rows_among_short_ones(ctx, gpu_device, d, dtype, out):
    """Rows of tens of thousands of entries, against 64-bit torch on the GPU by blocks of time; the bound is the definition's own,
    evaluated the same way."""
    lengths = [3, 30_011, 0, 17] + [5] * 200 + [20_000, 1, 0, 12_345]
    say(f"als_recur, als_recur_backward: rows of up to 30011 entries, d={d} {dtype} {out}")
    items = 300
    V, F = tables(items, d, dtype, 3)
    V[6] /= 1e10
    ptr, ids = history(lengths, items, 6)
    Y = csr(ptr, ids, items, gpu_device)
    last, states = als.als_recur(ctx, Y, V.to(gpu_device), F.to(gpu_device), all_states=True, dtype=out)
    want, want_states, bound, bound_states = ref.recur(ptr.numpy(), ids.numpy(), f64(V), f64(F))
    near(last, want, bound, out)
    near(states, want_states, bound_states, out)
    ds = (torch.randn(states.shape, generator=torch.Generator().manual_seed(5)) * 0.1).to(out)
    dV, dF, _ = als.als_recur_backward(ctx, Y, V.to(gpu_device), F.to(gpu_device), states, d_states=ds.to(gpu_device))
    want, bound = ref.recur_backward(ptr.numpy(), ids.numpy(), f64(V), f64(F), f64(states), f64(ds))
    near(dV, want[0], bound[0], out)
    near(dF, want[1], bound[1], out)


def test_many_rows(ctx, gpu_device):
    """Rows by the hundred thousand with stretches of empty ones, checked on a sample."""
    say("als_recur, als_recur_backward, als_sum_rows: 400000 rows")
    gen = torch.Generator().manual_seed(8)
    rows, items, d = 400_000, 5000, 32
    length = torch.randint(0, 6, (rows,), generator=gen)
    length[50_000:250_000] = 0
    length[-3000:] = 0
    length[1000] = 40_000
    ptr = torch.zeros(rows + 1, dtype=torch.int64)
    ptr[1:] = torch.cumsum(length, 0)
    n = int(ptr[-1])
    ids = torch.randint(-1, items, (n,), generator=gen).to(torch.int32)
    V, F = torch.randn((items, d), generator=gen), torch.randn((items, d), generator=gen)
    H0 = torch.randn((rows, d), generator=gen)
    Y = csr(ptr, ids, items, gpu_device)
    tv, tf, th = (t.to(gpu_device) for t in (V, F, H0))
    last, states = als.als_recur(ctx, Y, tv, tf, th, all_states=True)
    dl = torch.randn((rows, d), generator=gen)
    dV, dF, dH0 = als.als_recur_backward(ctx, Y, tv, tf, states, d_last=dl.to(gpu_device), H0=th)
    X = als.als_sum_rows(ctx, Y, tv)
    torch.cuda.synchronize()
    sample = torch.cat([torch.arange(990, 1010), torch.arange(49_990, 50_010), torch.arange(249_990, 250_200),
                        torch.randint(0, rows, (3000,), generator=gen), torch.arange(rows - 3010, rows - 2990), torch.tensor([rows - 1])])
    sub = torch.zeros(sample.numel() + 1, dtype=torch.int64)
    sub[1:] = torch.cumsum(length[sample], 0)
    at = torch.cat([torch.arange(int(ptr[r]), int(ptr[r + 1])) for r in sample])
    some, h0 = ids[at].numpy(), f64(H0[sample])
    want, want_states, bound, bound_states = ref.recur(sub.numpy(), some, f64(V), f64(F), h0)
    near(last[sample.to(gpu_device)], want, bound, F32)
    near(states[at.to(gpu_device)], want_states, bound_states, F32)
    want, bound = ref.recur_backward(sub.numpy(), some, f64(V), f64(F), f64(states[at.to(gpu_device)]), None, f64(dl[sample]), h0)
    for got, w, b, where in zip((dV, dF, dH0), want, bound, (at, at, sample)):
        near(got[where.to(gpu_device)], w, b, F32)
    want, bound = ref.sum_rows(sub.numpy(), some, None, f64(V))
    near(X[sample.to(gpu_device)], want, bound, F32)


def test_nothing_to_do(ctx, gpu_device):
    say("rows without entries, no rows, entries without items")
    d = 64
    V, F = (t.to(gpu_device) for t in tables(10, d, F32, 1))
    H0 = torch.randn((5, d), device=gpu_device)
    none = als.Csr(5, 10, torch.zeros(6, dtype=torch.int64, device=gpu_device), torch.zeros(0, dtype=torch.int32, device=gpu_device))
    last, states = als.als_recur(ctx, none, V, F, H0, all_states=True)
    assert torch.equal(last, H0) and states.shape == (0, d)
    assert torch.all(als.als_recur(ctx, none, V, F)[0] == 0)
    dV, dF, dH0 = als.als_recur_backward(ctx, none, V, F, states, d_last=H0, H0=H0)
    assert torch.equal(dH0, H0)
    assert torch.all(als.als_sum_rows(ctx, none, V) == 0)
    empty = als.Csr(0, 10, torch.zeros(1, dtype=torch.int64, device=gpu_device), torch.zeros(0, dtype=torch.int32, device=gpu_device))
    assert als.als_recur(ctx, empty, V, F)[0].shape == (0, d)
    assert als.als_sum_rows(ctx, empty, V).shape == (0, d)
    ids = torch.tensor([-1, 10, 55, -9], dtype=torch.int32, device=gpu_device)
    stray = als.Csr(2, 10, torch.tensor([0, 3, 4], device=gpu_device), ids)
    last, states = als.als_recur(ctx, stray, V, F, H0[:2], all_states=True)
    assert torch.equal(last, H0[:2]) and torch.equal(states, H0[[0, 0, 0, 1]])
    assert torch.all(als.als_sum_rows(ctx, stray, V) == 0)
    nowhere = als.Csr(2, 0, stray.indptr, ids)  # tables without rows
    last, _ = als.als_recur(ctx, nowhere, V[:0], F[:0], H0[:2])
    assert torch.equal(last, H0[:2])
    torch.cuda.synchronize()


def test_entries_outside_all_rows_stay_as_they_are(ctx, gpu_device):
    say("als_recur, als_recur_backward: entries before the first row and behind the last")
    d, items = 32, 20
    V, F = tables(items, d, F32, 1)
    ptr, ids = torch.tensor([3, 3, 10, 12]), torch.randint(0, items, (17,), generator=torch.Generator().manual_seed(1)).to(torch.int32)
    Y = csr(ptr, ids, items, gpu_device)
    states = torch.full((17, d), 7.0, device=gpu_device)
    last, _ = als.als_recur(ctx, Y, V.to(gpu_device), F.to(gpu_device), states=states)
    want, want_states, bound, bound_states = ref.recur(ptr.numpy(), ids.numpy(), f64(V), f64(F))
    near(last, want, bound, F32)
    near(states[3:12], want_states[3:12], bound_states[3:12], F32)
    grads = [torch.full((17, d), 7.0, device=gpu_device) for _ in range(2)]
    als.als_recur_backward(ctx, Y, V.to(gpu_device), F.to(gpu_device), states, d_states=states, out=(*grads, None))
    torch.cuda.synchronize()
    for t in [states] + grads:
        assert torch.all(t[:3] == 7.0) and torch.all(t[12:] == 7.0) and not torch.any(t[3:12] == 7.0)
    X = als.als_sum_rows(ctx, Y, V.to(gpu_device))
    want, bound = ref.sum_rows(ptr.numpy(), ids.numpy(), None, f64(V))
    near(X, want, bound, F32)


def test_values_that_are_not_finite_stay_in_their_row_and_column(ctx, gpu_device):
    say("als_recur: infinities and NaN")
    d = 16
    V, F = torch.ones((6, d)), torch.zeros((6, d))
    V[1, 2], V[2, 3], F[3, 4], F[4, 5], F[5, 6] = float("nan"), float("inf"), float("nan"), float("inf"), -float("inf")
    ptr, ids = torch.tensor([0, 70, 140, 340]), torch.zeros(340, dtype=torch.int32)
    ids[10:15] = torch.arange(1, 6, dtype=torch.int32)
    ids[200] = 1
    last, states = als.als_recur(ctx, csr(ptr, ids, 6, gpu_device), V.to(gpu_device), F.to(gpu_device), all_states=True)
    last, states = f64(last), f64(states)
    bad = np.zeros((3, d), dtype=bool)
    bad[0, [2, 3, 4]] = bad[2, 2] = True
    assert np.array_equal(~np.isfinite(last), bad)
    assert np.isposinf(last[0, 3]) and np.isnan(last[0, 2]) and np.isnan(last[0, 4])
    where = np.zeros(states.shape, dtype=bool)
    where[10:70, 2] = where[11:70, 3] = where[12:70, 4] = where[200:340, 2] = True
    assert np.array_equal(~np.isfinite(states), where)
    assert states[13, 5] == states[12, 5] and states[14, 6] == 1.0


def test_lists_that_are_not_in_order_stay_within_bounds(ctx, gpu_device):
    """indptr that falls, or points outside: every read and write stays in the buffers (the kernels clamp it), results aside."""
    say("als_recur, als_recur_backward, als_sum_rows: indptr out of order")
    d, items, n = 32, 9, 500
    V, F = (t.to(gpu_device) for t in tables(items, d, F32, 1))
    ids = torch.randint(0, items, (n,), generator=torch.Generator().manual_seed(2)).to(torch.int32)
    for ptr in ([0, 400, 100, 450, 500], [-50, 20, 700, 30, 500], [500, 400, 300, 0, 0], [2 ** 40, -2 ** 40, 3, 2 ** 62, 10]):
        Y = csr(torch.tensor(ptr), ids, items, gpu_device)
        big, last = padded(4, d, F32, gpu_device, 0, 7.0)
        big_states, states = padded(n, d, F32, gpu_device, 0, 7.0)
        grads = [padded(n, d, F32, gpu_device, 0, 7.0) for _ in range(2)]
        als.als_recur(ctx, Y, V, F, last=last, states=states)
        als.als_recur_backward(ctx, Y, V, F, states, d_states=states, out=(*[t for _, t in grads], None))
        als.als_sum_rows(ctx, Y, V, out=last)
        torch.cuda.synchronize()
        for whole, t in [(big, last), (big_states, states)] + grads:
            t.fill_(7.0)
            assert torch.all(whole == 7.0)


@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype,state", [(F32, F32), (BF16, F32), (F32, BF16), (BF16, BF16)])
def test_step_matches_the_definition(ctx, gpu_device, d, dtype, state):
    items = 40
    V, F = tables(items, d, dtype, 4)
    gen = torch.Generator().manual_seed(3)
    for rows in (1, 3, 64, 1000):
        say(f"als_recur_step d={d} {dtype} {state} rows={rows}")
        H = torch.randn((rows, d), generator=gen).to(state)
        ids = torch.randint(-2, items + 2, (rows,), generator=gen).to(torch.int32)
        parents = torch.randint(-1, rows + 1, (rows,), generator=gen).to(torch.int32)
        tv, tf = put(V, gpu_device, 8), put(F, gpu_device, 8)
        for p in (None, parents):
            at = np.arange(rows) if p is None else p.numpy()
            ok = (at >= 0) & (at < rows)
            before = np.where(ok[:, None], f64(H)[np.clip(at, 0, rows - 1)], 0.0)
            want, _, bound, _ = ref.recur(np.arange(rows + 1), ids.numpy(), f64(V), f64(F), before)
            X = als.als_recur_step(ctx, ids.to(gpu_device), tv, tf, H.to(gpu_device), None if p is None else p.to(gpu_device))
            torch.cuda.synchronize()
            near(X, want, bound, state)
            if p is None:  # in place
                X2 = put(H, gpu_device, 8)
                als.als_recur_step(ctx, ids.to(gpu_device), tv, tf, X2, out=X2)
                torch.cuda.synchronize()
                assert torch.equal(X2, X)
    # more rows than there are states: beams from one
    X = als.als_recur_step(ctx, torch.arange(5, dtype=torch.int32, device=gpu_device), tv, tf, H[:1].to(gpu_device),
                           torch.zeros(5, dtype=torch.int32, device=gpu_device))
    want, _, bound, _ = ref.recur(np.arange(6), np.arange(5), f64(V), f64(F), np.repeat(f64(H[:1]), 5, 0))
    near(X, want, bound, state)


def test_steps_are_the_recurrence(ctx, gpu_device):
    """Bound: both are within the definition's bound of it, so they differ by twice that."""
    say("als_recur_step after each other against als_recur")
    d, rows, steps, items = 64, 10, 40, 30
    V, F = (t.to(gpu_device) for t in tables(items, d, F32, 4))
    ids = torch.randint(0, items, (rows, steps), generator=torch.Generator().manual_seed(3)).to(torch.int32)
    ptr = torch.arange(0, rows * steps + 1, steps)
    last, _ = als.als_recur(ctx, csr(ptr, ids.view(-1), items, gpu_device), V, F)
    H = torch.zeros((rows, d), device=gpu_device)
    for t in range(steps):
        als.als_recur_step(ctx, ids[:, t].contiguous().to(gpu_device), V, F, H, out=H)
    _, _, bound, _ = ref.recur(ptr.numpy(), ids.view(-1).numpy(), f64(V), f64(F))
    assert np.all(np.abs(f64(last) - f64(H)) <= 2 * bound + 1e-37)


# ------------------------------------------------------------------------------------------------ sums

@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF16, F32), (F32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("lengths", [SHORT, LONG, [1], [0], [30_000, 3]], ids=["short", "long", "one", "none", "30000"])
def test_sum_rows_matches_the_definition(ctx, gpu_device, d, dtype, out, lengths):
    n = 70
    gen = torch.Generator().manual_seed(d)
    E = torch.randn((n, d), generator=gen).to(dtype)
    ptr, ids = history(lengths, n, len(lengths))
    for weighted, pad in ((False, 0), (True, 16)):
        say(f"als_sum_rows d={d} {dtype} -> {out}, {len(lengths)} rows of up to {max(lengths)}, weighted={weighted}")
        w = torch.randn(ids.numel(), generator=gen) if weighted else None
        want, bound = ref.sum_rows(ptr.numpy(), ids.numpy(), None if w is None else w.numpy(), f64(E))
        big, X = padded(len(lengths), d, out, gpu_device, pad, 7.0)
        als.als_sum_rows(ctx, csr(ptr, ids, n, gpu_device, w), put(E, gpu_device, pad), out=X)
        torch.cuda.synchronize()
        near(X, want, bound, out)
        X.fill_(7.0)
        assert torch.all(big == 7.0)


# ------------------------------------------------------------------------------------------------ clipping

def check_clip(ctx, tensors, bound, dev, place):
    """Norm: sums of squares in fp64, n additions; factor and product one rounding of fp32 each."""
    wide = [f64(t) for t in tensors]
    norm = np.sqrt(sum((w * w).sum() for w in wide))
    c = bound / norm if norm > bound and np.isfinite(norm) else 1.0
    if place == "strided":
        src = [put(t, dev, 3) if t.dim() == 2 and t.numel() else t.to(dev) for t in tensors]
    else:
        src = [t.to(dev) for t in tensors]
    kept = [t.clone() for t in src]
    out = None if place != "out" else [torch.full_like(t, 5.0) for t in src]
    got = als.als_clip(ctx, src, bound, out=out)
    torch.cuda.synchronize()
    n = sum(w.size for w in wide)
    if np.isfinite(norm):
        assert abs(float(got) - norm) <= (n + 4) * 2.0 ** -53 * norm
    else:
        assert np.array_equal(float(got), float(norm), equal_nan=True)
    for t, k, o, w in zip(src, kept, out or src, wide):
        if out is not None:
            assert torch.equal(t.view(torch.int16 if t.dtype is BF16 else torch.int32), k.view(torch.int16 if t.dtype is BF16 else torch.int32))
        if c == 1.0:
            assert np.array_equal(f64(o), w, equal_nan=True)
        else:
            near(o, w * c, 2.01 * ref.U * np.abs(w * c), t.dtype)


@pytest.mark.parametrize("place", ["in place", "out", "strided"])
@pytest.mark.parametrize("bound", [0.0, 1e-3, 7.0, 1e30, float("inf")])
def test_clip_matches_the_definition(ctx, gpu_device, place, bound):
    gen = torch.Generator().manual_seed(2)
    sets = {"one": [(1,)], "odd": [(3,), (4097,), (1, 1), (0,), (13, 77), (5, 0), (2, 3, 5), (100_003,)], "none": [], "many": [(k % 50 + 1, 7) for k in range(130)],
            "large": [(1000, 300), (2_000_003,)]}
    for name, shapes in sets.items():
        say(f"als_clip {name}, bound {bound}, {place}")
        tensors = [torch.randn(s, generator=gen).to((F32, BF16)[k % 2]) for k, s in enumerate(shapes)]
        check_clip(ctx, tensors, bound, gpu_device, place)


def test_clip_of_extreme_values(ctx, gpu_device):
    say("als_clip: values whose squares leave fp32's range, infinities, NaN, zeros")
    for size in (3e38, 1e30, 1e-30, 1e-41, 0.0):
        check_clip(ctx, [torch.full((5000,), size), torch.full((3, 5), size).to(BF16)], min(1.0, size), gpu_device, "out")
    for bad in (float("nan"), float("inf"), -float("inf")):
        x = torch.ones(10_000)
        x[7777] = bad
        check_clip(ctx, [torch.ones(3), x], 0.5, gpu_device, "in place")
        check_clip(ctx, [torch.ones(3), x], 0.5, gpu_device, "out")


# ------------------------------------------------------------------------------------------------ beams

def beam_case(groups, beams, k, seed, kind):
    gen = np.random.default_rng(seed)
    rows = groups * beams
    ids = gen.integers(0, 1000, (rows, k)).astype(np.int32)
    scores = np.sort(gen.normal(size=(rows, k)).astype(np.float32), 1)[:, ::-1].copy()
    kw = dict(lse=gen.normal(size=rows).astype(np.float32), totals=gen.normal(size=rows).astype(np.float32))
    if kind == "ties":
        scores = np.round(scores * 2) / 2
        kw = dict(lse=np.zeros(rows, dtype=np.float32), totals=np.round(kw["totals"]))
        scores[:, -1] = -0.0
    if kind == "first":
        kw["totals"] = None
    if kind == "few":
        ids[gen.random(ids.shape) < 0.9] = -1
        kw["totals"][gen.random(rows) < 0.5] = -np.inf
    if kind == "none":
        ids[:] = -1
    if kind == "odd":
        scores[gen.random(scores.shape) < 0.2] = np.nan
        scores[gen.random(scores.shape) < 0.1] = -np.inf
        scores[gen.random(scores.shape) < 0.05] = np.inf
        kw["lse"][gen.random(rows) < 0.2] = np.nan
        kw["lse"][gen.random(rows) < 0.2] = -np.inf
    if kind in ("ended", "factors", "all ended"):
        kw["last"] = np.where(gen.random(rows) < (2 if kind == "all ended" else 0.4), 0, 7).astype(np.int32)
        kw["end"] = 0
    if kind == "factors":
        kw["lengths"] = gen.integers(0, 9, rows).astype(np.int32)
        kw["factors"] = (1.0 / (1 + np.arange(6))).astype(np.float32)
    return ids, np.ascontiguousarray(scores, dtype=np.float32), kw


@pytest.mark.parametrize("kind", ["plain", "ties", "first", "few", "none", "odd", "ended", "all ended", "factors"])
@pytest.mark.parametrize("groups,beams,k", [(1, 1, 1), (1, 8, 8), (3, 5, 7), (2, 64, 64), (7, 50, 64), (5, 64, 3), (40, 4, 64), (3, 1, 64), (300, 2, 2)])
def test_beam_matches_the_definition(ctx, gpu_device, groups, beams, k, kind):
    say(f"als_beam {groups} x {beams} x {k} {kind}")
    ids, scores, kw = beam_case(groups, beams, k, 7, kind)
    want = ref.beam(ids, scores, beams=beams, temperature=0.7, **kw)
    dev = {n: torch.from_numpy(v).to(gpu_device) if isinstance(v, np.ndarray) else v for n, v in kw.items()}
    got = als.als_beam(ctx, torch.from_numpy(ids).to(gpu_device), torch.from_numpy(scores).to(gpu_device), beams=beams, temperature=0.7, **dev)
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert np.array_equal(g.cpu().numpy(), w)


@pytest.mark.parametrize("beams,groups", [(1, 7), (2, 3), (5, 40), (8, 1), (32, 3), (64, 2), (50, 11), (3, 700)])
def test_reorder_moves_every_element(ctx, gpu_device, beams, groups):
    rows = beams * groups
    gen = torch.Generator().manual_seed(beams)
    local = torch.randint(0, beams, (rows,), generator=gen)
    parents = (torch.arange(rows) // beams * beams + local).to(torch.int32)
    parents[rows // 2] = -1
    parents[0] = rows if groups > 1 else 2 ** 31 - 1  # not of this group
    keep = torch.rand(rows, generator=gen) < 0.3
    parents[keep] = torch.arange(rows, dtype=torch.int32)[keep]
    word = lambda *s: torch.randint(-2 ** 31, 2 ** 31, (rows,) + s, generator=gen, dtype=torch.int64).to(torch.int32)  # noqa: E731
    states = [torch.randn((rows, 64), generator=gen), word(1), word(3), word(50), word(1031), word(4, 5, 7).to(torch.int64) << 9,
              word(7).to(torch.int16), word(129).to(torch.int16).view(BF16), word(), torch.randn((rows, 0))]
    from_row = parents.long()
    ok = (from_row >= 0) & (from_row < rows) & (from_row.clamp(0, rows - 1) // beams == torch.arange(rows) // beams)
    want = [torch.where(ok.view([-1] + [1] * (t.dim() - 1)), t.view(torch.int16)[from_row.clamp(0, rows - 1)] if t.dtype is BF16 else t[from_row.clamp(0, rows - 1)],
                        torch.zeros((), dtype=torch.int16 if t.dtype is BF16 else t.dtype)) for t in states]
    bits = lambda t: t.cpu().view(torch.int16) if t.dtype is BF16 else t.cpu()  # noqa: E731
    p = parents.to(gpu_device)
    say(f"als_reorder {groups} groups of {beams}, to other buffers")
    src = [t.to(gpu_device) for t in states]
    out = als.als_reorder(ctx, p, beams, src, out=[torch.full_like(t, 3) for t in src])
    torch.cuda.synchronize()
    for g, w, s, t in zip(out, want, src, states):
        assert torch.equal(bits(g), w) and torch.equal(bits(s), bits(t))
    say(f"als_reorder {groups} groups of {beams}, in place")
    als.als_reorder(ctx, p, beams, src)
    torch.cuda.synchronize()
    for g, w in zip(src, want):
        assert torch.equal(bits(g), w)
    say(f"als_reorder {groups} groups of {beams}, rows of wider matrices, many states")
    wide = [torch.full((rows, 40), 9, dtype=torch.int32, device=gpu_device) for _ in range(40)]
    small = [w[:, k % 30:k % 30 + 7] for k, w in enumerate(wide)]
    for k, s in enumerate(small):
        s.copy_(states[3][:, :7] + k)
    als.als_reorder(ctx, p, beams, small)
    torch.cuda.synchronize()
    for k, (s, w) in enumerate(zip(small, wide)):
        assert torch.equal(s.cpu(), torch.where(ok[:, None], states[3][from_row.clamp(0, rows - 1)][:, :7] + k, 0))
        s.fill_(9)
        assert torch.all(w == 9)


# ------------------------------------------------------------------------------------------------ together

def session(ctx, Y, V, F, T, beams, steps, k, end=0):
    """Sessions continued by `steps` items: scores of all beams against a 4-bit table, each beam's best, the best of each group."""
    groups, items, dev = Y.rows, V.shape[0], V.device
    H = als.als_recur(ctx, Y, V, F)[0].repeat_interleave(beams, 0)
    rows = groups * beams
    seq = torch.full((rows, steps), -1, dtype=torch.int32, device=dev)
    totals = last = None
    lengths = torch.zeros(rows, dtype=torch.int32, device=dev)
    for t in range(steps):
        S = als.als_scores(ctx, H, T)
        ids, scores, lse = als.als_select(ctx, S, k, temperature=0.5)
        parents, last, totals, lengths = als.als_beam(ctx, ids, scores, lse, totals, beams, 0.5, last, end, lengths)
        als.als_reorder(ctx, parents, beams, [seq])
        seq[:, t] = last
        H = als.als_recur_step(ctx, last, V, F, H, parents)
    return seq, totals, lengths, H


def test_a_session_on_a_stream_and_in_a_graph(ctx, gpu_device):
    """The same bits live, on another stream and replayed; beams' totals are sums of log-probabilities along their own sequences:
    recomputed from the table in 64 bits, off by fp32's roundings of scores (128 products), sums and exponents."""
    say("als_recur, als_scores, als_select, als_beam, als_reorder, als_recur_step: a session")
    gen = torch.Generator().manual_seed(12)
    items, d, groups, beams, steps, k = 3001, 64, 5, 6, 4, 6
    V, F = torch.randn((items, d), generator=gen).to(gpu_device), torch.randn((items, d), generator=gen).to(gpu_device)
    T = als.als_quantize(ctx, V)
    ptr, ids = history([3, 0, 40, 200, 1], items, 2, stray=False)
    Y = csr(ptr, ids, items, gpu_device)
    want = session(ctx, Y, V, F, T, beams, steps, k)
    torch.cuda.synchronize()
    seq, totals, lengths, H = (t.cpu() for t in want)
    Tv, hv, fv = f64(als.als_dequantize(ctx, T)), f64(V), f64(F)
    start, _, _, _ = ref.recur(ptr.numpy(), ids.numpy(), hv, fv)
    for r in range(groups * beams):
        h, total, over = start[r // beams], 0.0, False
        for t in range(steps):
            i = int(seq[r, t])
            if over:
                assert i == 0
            else:
                x = (Tv @ h) / 0.5
                total += x[i] - x.max() - np.log(np.exp(x - x.max()).sum())
            h = ref.recur([0, 1], [i], hv, fv, h[None])[0][0]
            over = over or i == 0
        assert abs(total - float(totals[r])) <= 1e-3
        assert int(lengths[r]) == (seq[r].tolist().index(0) + 1 if 0 in seq[r].tolist() else steps)
        assert np.allclose(h, f64(H[r]), atol=1e-4)
    assert torch.all(totals.view(groups, beams)[:, :-1] >= totals.view(groups, beams)[:, 1:])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = session(ctx, Y, V, F, T, beams, steps, k)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = session(ctx, Y, V, F, T, beams, steps, k)
    for step in range(4):
        V.copy_(torch.randn((items, d), generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        again = [t.clone() for t in out]
        for a, b in zip(again, session(ctx, Y, V, F, T, beams, steps, k)):
            assert torch.equal(a, b)


def train(ctx, Y, by_item, V, F, target, bound):
    """Gradients of |last - target|^2 / 2 with respect to both tables, clipped together."""
    last, states = als.als_recur(ctx, Y, V, F, all_states=True)
    dV, dF, _ = als.als_recur_backward(ctx, Y, V, F, states, d_last=last - target)
    grads = [als.als_sum_rows(ctx, by_item, t) for t in (dV, dF)]
    norm = als.als_clip(ctx, grads, bound)
    return grads[0], grads[1], norm


def test_training_gradients_live_and_in_a_graph(ctx, gpu_device):
    say("als_recur, als_recur_backward, als_sum_rows, als_clip: gradients of a training step")
    gen = torch.Generator().manual_seed(3)
    items, d, rows = 200, 32, 300
    V, F = torch.randn((items, d), generator=gen), torch.randn((items, d), generator=gen)
    ptr, ids = history([int(x) for x in torch.randint(0, 60, (rows,), generator=gen)] + [5000], items, 5, stray=False)
    n, target = ids.numel(), torch.randn((rows + 1, d), generator=gen)
    order = torch.argsort(ids, stable=True).to(torch.int32)
    heads = torch.zeros(items + 1, dtype=torch.int64)
    heads[1:] = torch.cumsum(torch.bincount(ids.long(), minlength=items), 0)
    Y, by_item = csr(ptr, ids, items, gpu_device), csr(heads, order, n, gpu_device)
    dev = [t.to(gpu_device) for t in (V, F, target)]
    got = train(ctx, Y, by_item, *dev, 1.0)
    torch.cuda.synchronize()
    last, states, _, _ = ref.recur(ptr.numpy(), ids.numpy(), f64(V), f64(F))
    (dV, dF, _), _ = ref.recur_backward(ptr.numpy(), ids.numpy(), f64(V), f64(F), states, d_last=last - f64(target))
    gV, gF = np.zeros((items, d)), np.zeros((items, d))
    np.add.at(gV, ids.numpy(), dV)
    np.add.at(gF, ids.numpy(), dF)
    norm = np.sqrt((gV ** 2).sum() + (gF ** 2).sum())
    assert norm > 1 and abs(float(got[2]) - norm) <= 1e-4 * norm
    for g, w in zip(got, (gV, gF)):
        assert np.linalg.norm(f64(g) - w / norm) <= 1e-4 * np.linalg.norm(w / norm)
    for a, b in zip(got, train(ctx, Y, by_item, *dev, 1.0)):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = train(ctx, Y, by_item, *dev, 1.0)
    for _ in range(4):
        dev[0].add_(0.1)
        graph.replay()
        torch.cuda.synchronize()
        again = [t.clone() for t in out]
        for a, b in zip(again, train(ctx, Y, by_item, *dev, 1.0)):
            assert torch.equal(a, b)


def test_same_bits_every_time(ctx, gpu_device):
    say("als_recur, als_recur_backward, als_sum_rows, als_clip, als_beam: the same bits on every call")
    V, F = (t.to(gpu_device) for t in tables(100, 64, F32, 4))
    ptr, ids = history([20_000, 5, 0, 300] + [7] * 3000, 100, 5)
    Y = csr(ptr, ids, 100, gpu_device)

    def calls():
        last, states = als.als_recur(ctx, Y, V, F, all_states=True)
        grads = als.als_recur_backward(ctx, Y, V, F, states, d_states=states)[:2]
        X = als.als_sum_rows(ctx, Y, V)
        out = [torch.empty_like(t) for t in (last, states)]
        return [last, states, *grads, X, als.als_clip(ctx, [last, states], 1.0, out=out), *out]

    first = calls()
    for _ in range(4):
        for a, b in zip(first, calls()):
            assert torch.equal(a, b)


def test_refusals(ctx, gpu_device):
    say("what the operators over ordered histories refuse")
    dev, z = gpu_device, torch.zeros

    def refused(status, f, *args, **kw):
        with pytest.raises(als.AlsError) as e:
            f(ctx, *args, **kw)
        assert e.value.status == status

    V, F = z((10, 32), device=dev), z((10, 32), device=dev)
    Y = als.Csr(2, 10, torch.tensor([0, 3, 5], device=dev), z(5, dtype=torch.int32, device=dev))
    refused(als.ALS_EDTYPE, als.als_recur, Y, V, F.to(BF16))
    refused(als.ALS_EDTYPE, als.als_recur, Y, z((10, 48), device=dev), z((10, 48), device=dev))
    refused(als.ALS_ESHAPE, als.als_recur, Y, V, F[:9])
    refused(als.ALS_ESHAPE, als.als_recur, als.Csr(2, 9, Y.indptr, Y.indices), V, F)
    refused(als.ALS_ESHAPE, als.als_recur, Y, V, F, H0=z((3, 32), device=dev))
    refused(als.ALS_ESHAPE, als.als_recur, Y, V, F, states=z((4, 32), device=dev))
    refused(als.ALS_ESHAPE, als.als_recur, Y, V, F, last=z((2, 64), device=dev))
    refused(als.ALS_EALIAS, als.als_recur, Y, V, F, last=V[:2])
    both = z((12, 32), device=dev)
    refused(als.ALS_EALIAS, als.als_recur, Y, V, F, last=both[4:6], states=both[:5])
    refused(als.ALS_EALIAS, als.als_recur, Y, V, F, H0=both[:2], last=both[:2])
    c, tv, tl = als._table(both[:5]), als._table(V), None
    import ctypes
    y = Y.c()
    lib = ctx.lib
    assert lib.als_recur(ctx.handle, ctypes.byref(y), ctypes.byref(tv), ctypes.byref(tv), None, None, None, None) == als.ALS_EINVAL
    assert lib.als_recur(ctx.handle, ctypes.byref(y), ctypes.byref(tv), ctypes.byref(tv), None, ctypes.byref(c), tl, None) == als.ALS_OK  # states alone
    loose = als.c_als_csr(2, 4, 5, Y.indptr.data_ptr(), None, None)  # more entries than table rows, and no ids
    t4 = als._table(V[:4])
    assert lib.als_recur(ctx.handle, ctypes.byref(loose), ctypes.byref(t4), ctypes.byref(t4), None, None, ctypes.byref(als._table(both[:2])), None) == als.ALS_ESHAPE
    refused(als.ALS_EINVAL, als.als_solve_rows, als.Csr(2, 10, torch.tensor([0, 3, 10], device=dev), None), V, z((32, 32), device=dev), als.make_params(0.1, 0.1), z((2, 32), device=dev))
    refused(als.ALS_EINVAL, als.als_sum_rows, als.Csr(2, 10, torch.tensor([0, 3, 10], device=dev), None), V)
    items = z(2, dtype=torch.int32, device=dev)
    refused(als.ALS_ESHAPE, als.als_recur_step, items, V, F, z((3, 32), device=dev))
    refused(als.ALS_EALIAS, als.als_recur_step, items, V, F, both[:2], parents=items, out=both[:2])
    refused(als.ALS_EALIAS, als.als_recur_step, items, V, F, both[:2], out=both[1:3])
    refused(als.ALS_ESHAPE, als.als_recur_step, items, V, F, z((2, 64), device=dev))
    s = z((5, 32), device=dev)
    refused(als.ALS_EINVAL, als.als_recur_backward, Y, V, F, s)
    refused(als.ALS_EDTYPE, als.als_recur_backward, Y, V, F, s, d_states=s.to(BF16))
    refused(als.ALS_EDTYPE, als.als_recur_backward, Y, V, F, s, d_states=s, dtype=BF16)
    refused(als.ALS_ESHAPE, als.als_recur_backward, Y, V, F, s[:4], d_last=s[:2])
    refused(als.ALS_EALIAS, als.als_recur_backward, Y, V, F, s, d_states=s, out=(both[:5], both[4:9], None))
    refused(als.ALS_EALIAS, als.als_recur_backward, Y, V, F, s, d_states=both[:5], out=(both[:5], both[5:10], None))
    refused(als.ALS_ESHAPE, als.als_sum_rows, Y, V, out=z((3, 32), device=dev))
    refused(als.ALS_EALIAS, als.als_sum_rows, Y, V, out=V[:2])
    for bad in (-1.0, float("nan")):
        refused(als.ALS_EINVAL, als.als_clip, [V], bad)
    refused(als.ALS_EALIAS, als.als_clip, [V, V], 1.0)
    refused(als.ALS_EALIAS, als.als_clip, [both[:4]], 1.0, out=[both[2:6]])
    refused(als.ALS_EALIAS, als.als_clip, [both[:4], both[4:8]], 1.0, out=[both[4:8], both[:4]])
    refused(als.ALS_EDTYPE, als.als_clip, [V], 1.0, out=[V.to(BF16)])
    ids, scores, per = z((4, 3), dtype=torch.int32, device=dev), z((4, 3), device=dev), z(4, device=dev)
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        refused(als.ALS_EINVAL, als.als_beam, ids, scores, per, per, 2, temperature=bad)
    refused(als.ALS_EINVAL, als.als_beam, z((130, 3), dtype=torch.int32, device=dev), z((130, 3), device=dev), None, None, 65)
    refused(als.ALS_EINVAL, als.als_beam, z((4, 65), dtype=torch.int32, device=dev), z((4, 65), device=dev), None, None, 2)
    parents = z(4, dtype=torch.int32, device=dev)
    refused(als.ALS_EALIAS, als.als_reorder, parents, 2, [scores, scores])
    refused(als.ALS_EALIAS, als.als_reorder, parents, 2, [parents])
    refused(als.ALS_EALIAS, als.als_reorder, parents, 2, [both[:4]], out=[both[1:5]])
    refused(als.ALS_EINVAL, als.als_reorder, parents, 2, [z((4, 2), device=dev) for _ in range(65)])
    refused(als.ALS_EINVAL, als.als_reorder, z(130, dtype=torch.int32, device=dev), 65, [])
    torch.cuda.synchronize()
