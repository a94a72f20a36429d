"""Infinities and NaN in ordered histories: they stay in their row and column (a gradient's in its entry and those before it), also
where rows are cut into pieces.  Against the 64-bit references: the same elements are not finite, and the others are within bounds."""
import numpy as np
import pytest
import torch

import history_ref as ref
from gpu_util import f64, say
from paper_2112_02194_amd import binding as als
from test_gpu_history import BF16, F32, csr, stored

pytestmark = pytest.mark.gpu
LENGTHS = [3000, 5, 0, 700, 40, 9000, 1, 64]
KINDS = [(16, F32), (64, BF16), (128, F32)]


@pytest.fixture(scope="module")
def ctx(gpu_device):
    c = als.Context(0)
    yield c
    c.close()


def lists(seed):
    """Items 0 .. 19 are ordinary, some entries have none; items 20, 21, 22, 23 stand where the tests put them."""
    gen = torch.Generator().manual_seed(seed)
    ptr = torch.tensor(np.concatenate([[0], np.cumsum(LENGTHS)]))
    ids = torch.randint(-1, 20, (sum(LENGTHS),), generator=gen).to(torch.int32)
    for item, rows in ((20, (0, 4, 5)), (21, (3, 5)), (22, (0, 5, 7)), (23, (1, 3))):
        for row in rows:
            ids[ptr[row] + (item * 131 + row * 977) % LENGTHS[row]] = item
    return ptr, ids


def tables(d, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    V, F = torch.randn((24, d), generator=gen), 1.5 + torch.randn((24, d), generator=gen)
    return V.to(dtype), F.to(dtype)


def same(got, want, bound, dtype):
    got, there = f64(got), np.isfinite(want)
    assert np.array_equal(np.isfinite(got), there)
    assert np.all(np.abs(got[there] - want[there]) <= stored(bound[there], want[there], dtype))


@pytest.mark.parametrize("d,dtype", KINDS)
def test_recurrence(ctx, gpu_device, d, dtype):
    say(f"als_recur: infinities and NaN, rows of up to {max(LENGTHS)}, d={d} {dtype}")
    ptr, ids = lists(1)
    V, F = tables(d, dtype, 2)
    V[20, 2], V[21, 3], F[22, 5], V[23, 6] = float("nan"), float("inf"), float("nan"), -float("inf")
    H0 = torch.randn((len(LENGTHS), d), generator=torch.Generator().manual_seed(3))
    H0[1, 7], H0[5, 8] = float("nan"), float("inf")
    with np.errstate(invalid="ignore"):
        want, want_states, bound, bound_states = ref.recur(ptr.numpy(), ids.numpy(), f64(V), f64(F), f64(H0))
    Y = csr(ptr, ids, 24, gpu_device)
    last, states = als.als_recur(ctx, Y, V.to(gpu_device), F.to(gpu_device), H0.to(gpu_device), all_states=True)
    alone, _ = als.als_recur(ctx, Y, V.to(gpu_device), F.to(gpu_device), H0.to(gpu_device))
    torch.cuda.synchronize()
    same(last, want, bound, F32)
    same(alone, want, bound, F32)
    same(states, want_states, bound_states, F32)


@pytest.mark.parametrize("d,dtype", KINDS)
def test_gradients(ctx, gpu_device, d, dtype):
    say(f"als_recur_backward: infinities and NaN, rows of up to {max(LENGTHS)}, d={d} {dtype}")
    ptr, ids = lists(1)
    V, F = tables(d, dtype, 2)
    n, gen = ids.numel(), torch.Generator().manual_seed(4)
    states, ds, dl = (torch.randn((k, d), generator=gen) for k in (n, n, len(LENGTHS)))
    V[20, 2], F[22, 5] = float("nan"), float("nan")
    ds[2500, 3], ds[int(ptr[5]) + 6000, 4], dl[3, 6], dl[0, 7] = float("nan"), float("inf"), float("nan"), -float("inf")
    states[1200, 8], states[int(ptr[5]) + 10, 9] = float("nan"), float("inf")
    H0 = torch.randn((len(LENGTHS), d), generator=gen)
    H0[5, 10] = float("nan")
    dev = [t.to(gpu_device) for t in (V, F, states, ds, dl, H0)]
    got = als.als_recur_backward(ctx, csr(ptr, ids, 24, gpu_device), *dev)
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        want, bound = ref.recur_backward(ptr.numpy(), ids.numpy(), f64(V), f64(F), f64(states), f64(ds), f64(dl), f64(H0))
    none = (ids < 0).numpy()[:, None]
    for k in (0, 1):  # zeros where there is no item, whatever comes by
        want[k][np.broadcast_to(none, want[k].shape)] = 0.0
        bound[k][np.broadcast_to(none, want[k].shape)] = 0.0
    for g, w, b in zip(got, want, bound):
        same(g, w, b, F32)


@pytest.mark.parametrize("d,dtype", KINDS)
@pytest.mark.parametrize("weighted", [False, True])
def test_sums(ctx, gpu_device, d, dtype, weighted):
    say(f"als_sum_rows: infinities and NaN, rows of up to {max(LENGTHS)}, d={d} {dtype}, weighted={weighted}")
    ptr, ids = lists(1)
    E, _ = tables(d, dtype, 2)
    E[20, 2], E[21, 3], E[22, 3], E[23, 6] = float("nan"), float("inf"), -float("inf"), -float("inf")
    w = torch.rand(ids.numel(), generator=torch.Generator().manual_seed(5)) + 0.5 if weighted else None
    if weighted:
        w[ids < 0] = float("nan")  # of entries without an item: not looked at
        w[int(ptr[3]) + 5] = float("inf")
        ids[int(ptr[3]) + 5] = 1
    X = als.als_sum_rows(ctx, csr(ptr, ids, 24, gpu_device, w), E.to(gpu_device))
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        want, bound = ref.sum_rows(ptr.numpy(), ids.numpy(), None if w is None else w.numpy(), f64(E))
    same(X, want, bound, F32)
    inf = np.isinf(want)  # an infinity without another of the other sign is the sum
    assert np.array_equal(f64(X)[inf], want[inf])


@pytest.mark.parametrize("d,dtype", KINDS)
def test_infinite_states_pass_entries_without_items(ctx, gpu_device, d, dtype):
    """Nothing takes part of them, whatever groups, stages and pieces they cross; and gates that keep nearly all keep an infinity."""
    say(f"als_recur, als_recur_step: infinite first states, d={d} {dtype}")
    V, F = tables(d, dtype, 2)
    F[0] = 12.0
    H0 = torch.full((len(LENGTHS), d), float("inf"))
    H0[:, 1::2] = -float("inf")
    ptr, ids = lists(1)
    for item in (-1, 0):
        ids[:] = item
        Y = csr(ptr, ids, 24, gpu_device)
        last, states = als.als_recur(ctx, Y, V.to(gpu_device), F.to(gpu_device), H0.to(gpu_device), all_states=True)
        alone, _ = als.als_recur(ctx, Y, V.to(gpu_device), F.to(gpu_device), H0.to(gpu_device))
        step = als.als_recur_step(ctx, Y.indices[:len(LENGTHS)], V.to(gpu_device), F.to(gpu_device), H0.to(gpu_device))
        torch.cuda.synchronize()
        for got in (last, alone, step):
            assert torch.equal(got.cpu(), H0)
        assert torch.equal(states.cpu(), H0.repeat_interleave(torch.tensor(LENGTHS), 0))
