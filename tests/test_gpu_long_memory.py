"""Ordered histories whose gates keep for thousands of entries: one item over and over, so that an error of its gate counts every time.

With one item in every entry the states have a closed form: s^t by exp(t log s), log s = -log1p(exp(-F)) in 64 bits, and
    h_t = x + (h_0 - x) s^t,    g_j = d (1 - s^(j+1)) / (1 - s) + s^j d_last, j entries before the last one.

Bounds, u = 2^-24, m the largest magnitude on the way: what comes into an entry was rounded once for every join on its way, not once
for every entry of the row.  A row of 65 537 entries lies in 512 to 2100 chunks of 32 to 128 entries; of a chunk's entries a lane walks at
most 40 one after the other and joins 4 to 8 groups or tiles; of the chunks' maps a lane joins at most 33 one after the other, and 128 such
stretches.  An entry or a join is two roundings of the state, and two of the share that its map keeps or gives away, relative to that
share: 4 u m; within the 40, where gates are multiplied as they are, a gate near 1 is off by up to 3 u besides (its sum, its
reciprocal): 40 * 7 + (8 + 33 + 128) * 4 = 956, below 4 * 240.  1 - s itself is off by (1.5 |F| + 7) u of its size (history_ref), which
over a row's entries changes a state by that much of m at most.  So a state is off by (4 * 240 + 1.5 |F| + 7) u m; a gate near 1 that is
off by u / 2 once an entry would make that 65 537 u / 2 and more."""
import numpy as np
import pytest
import torch

import history_ref as ref
from gpu_util import f64, say
from paper_2112_02194_amd import binding as als
from test_gpu_history import BF16, F32

pytestmark = pytest.mark.gpu
LENGTHS = [5, 65_537, 0, 20_000, 1]
GATES = [6.0, 8.0, 10.0, 12.0, 14.0, 3.0, 2.0, 1.0]
ROUNDINGS = 4 * 240


@pytest.fixture(scope="module")
def ctx(gpu_device):
    c = als.Context(0)
    yield c
    c.close()


def one_item(d, dtype):
    F = torch.tensor(GATES * (d // 8)).view(1, d)
    V = torch.tensor([1.0, -1.0, 0.75] * 43)[:d].view(1, d)
    return V.to(dtype), F.to(dtype)


def powers(F, t):
    return np.exp(-t[:, None] * np.log1p(np.exp(-F)))


@pytest.mark.parametrize("d,dtype", [(16, F32), (32, BF16), (64, F32), (128, F32), (128, BF16)])
def test_states(ctx, gpu_device, d, dtype):
    say(f"als_recur: one item {max(LENGTHS)} times, d={d} {dtype}")
    V, F = one_item(d, dtype)
    x, f, rows, n = f64(V), f64(F), len(LENGTHS), sum(LENGTHS)
    ptr = torch.tensor(np.concatenate([[0], np.cumsum(LENGTHS)]))
    Y = als.Csr(rows, 1, ptr.to(gpu_device), torch.zeros(n, dtype=torch.int32, device=gpu_device))
    H0 = torch.full((rows, d), -0.5)
    bound = 1.01 * (ROUNDINGS + 1.5 * np.abs(f) + 7) * ref.U  # m = 1
    last, states = als.als_recur(ctx, Y, V.to(gpu_device), F.to(gpu_device), H0.to(gpu_device), all_states=True)
    alone, _ = als.als_recur(ctx, Y, V.to(gpu_device), F.to(gpu_device), H0.to(gpu_device))
    want = x + (-0.5 - x) * powers(f, np.array(LENGTHS, dtype=np.float64))
    for got in (last, alone):
        worst = (np.abs(f64(got) - want) / bound).max(0)[:8]
        print("last", worst)
        assert np.all(worst <= 1)
    t = np.concatenate([np.arange(1.0, k + 1) for k in LENGTHS])
    worst = (np.abs(f64(states) - (x + (-0.5 - x) * powers(f, t))) / bound).max(0)[:8]
    print("states", worst)
    assert np.all(worst <= 1)


@pytest.mark.parametrize("d,dtype", [(16, F32), (32, BF16), (64, F32), (128, F32), (128, BF16)])
def test_gradients(ctx, gpu_device, d, dtype):
    say(f"als_recur_backward: one item {max(LENGTHS)} times, d={d} {dtype}")
    V, F = one_item(d, dtype)
    x, f, rows, n = f64(V), f64(F), len(LENGTHS), sum(LENGTHS)
    ptr = torch.tensor(np.concatenate([[0], np.cumsum(LENGTHS)]))
    Y = als.Csr(rows, 1, ptr.to(gpu_device), torch.zeros(n, dtype=torch.int32, device=gpu_device))
    H0 = torch.full((rows, d), -0.5)
    t = np.concatenate([np.arange(1.0, k + 1) for k in LENGTHS])
    states = torch.from_numpy(x + (-0.5 - x) * powers(f, t)).float()
    d_each, d_last = 2.0 ** -12, 0.5
    dev = [a.to(gpu_device) for a in (V, F, states, torch.full((n, d), d_each), torch.full((rows, d), d_last), H0)]
    dV, dF, dH0 = als.als_recur_backward(ctx, Y, dev[0], dev[1], dev[2], dev[3], dev[4], dev[5])
    keep, take = 1 / (1 + np.exp(-f)), np.exp(-f) / (1 + np.exp(-f))
    behind = np.concatenate([np.arange(k - 1, -1, -1.0) for k in LENGTHS])
    g = d_each * (1 - powers(f, behind + 1)) / take + powers(f, behind) * d_last
    m = np.minimum(d_each / take, d_each * max(LENGTHS)) + d_last  # of all that is added up
    gate = (1.5 * np.abs(f) + 7) * ref.U
    bound = 1.01 * (ROUNDINGS * ref.U + gate) * m
    k = np.array(LENGTHS, dtype=np.float64)
    want = d_each * keep * (1 - powers(f, k)) / take + powers(f, k) * d_last  # s g of a row's first entry
    worst = [(np.abs(f64(dH0) - want) / bound).max(0)[:8]]
    worst.append((np.abs(f64(dV) - take * g) / (take * (bound + 1.01 * (gate + ref.U) * m))).max(0)[:8])
    before = np.concatenate([np.full((1, d), -0.5), f64(states)[:-1]])
    before[np.cumsum([0] + LENGTHS[:-1])[np.array(LENGTHS) > 0]] = -0.5
    size = np.abs(before - x)
    want = g * (before - x) * keep * take
    # a difference, rounded relative to itself, times two gates
    worst.append((np.abs(f64(dF) - want) / (keep * take * size * (bound + 1.01 * (2 * gate + 4 * ref.U) * m) + ref.TINY)).max(0)[:8])
    for name, w in zip(("dH0", "dV", "dF"), worst):
        print(name, w)
    for w in worst:
        assert np.all(w <= 1)


def test_steps(ctx, gpu_device):
    """One rounding of the state a step, so 4096 of them may be off by 4096 u at F = 9; the factor 1 - s is as exact as its own bits
    there, which shows where the state comes from below: h_t - h_(t-1) = (1 - s) (x - h_(t-1)), a step of the state off at most."""
    say("als_recur_step: one item 300 times")
    d = 16
    V, F = one_item(d, F32)
    x, f = f64(V), f64(F)
    items = torch.zeros(1, dtype=torch.int32, device=gpu_device)
    H = torch.full((1, d), -0.5, device=gpu_device)
    tv, tf = V.to(gpu_device), F.to(gpu_device)
    take = np.exp(-f) / (1 + np.exp(-f))
    for _ in range(300):
        before = f64(H)
        H = als.als_recur_step(ctx, items, tv, tf, H)
        want = before + take * (x - before)
        # half a step of the state, and what is added is off by its gate's error and three roundings
        bound = ref.U * np.abs(want) + ((1.5 * np.abs(f) + 7) + 4) * ref.U * take * (np.abs(x) + np.abs(before))
        assert np.all(np.abs(f64(H) - want) <= 1.01 * bound)
