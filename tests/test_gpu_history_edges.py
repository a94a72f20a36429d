"""Ordered histories on the GPU where it is easy to go wrong: offsets beyond 32 bits, rows around every border of the kernels' chunks
and stages, recordings that share a workspace, what the C interface allows beside the binding.

Bounds are history_ref's."""
import ctypes

import numpy as np
import pytest
import torch

import history_ref as ref
from gpu_util import f64, say
from paper_2112_02194_amd import binding as als
from test_gpu_history import BF16, F32, csr, history, near, tables

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(gpu_device):
    c = als.Context(0)
    yield c
    c.close()


def wide(t):
    return t.cpu().to(torch.float64)


def apart(t, dev, ld):
    """The same rows `ld` elements apart, the space between them as it comes."""
    rows, d = t.shape
    big = torch.empty((rows - 1) * ld + d, dtype=t.dtype, device=dev)
    out = big.as_strided((rows, d), (ld, 1))
    out.copy_(t.to(dev))
    return out


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_far_apart(ctx, gpu_device, dtype):
    """Offsets beyond 2^32 bytes in every table."""
    d, items, ld = 32, 12, (1 << 28) + 16
    say(f"als_recur, als_recur_backward, als_recur_step, als_sum_rows: rows {ld} elements apart, {dtype}")
    V, F = tables(items, d, dtype, 1)
    V[6] = 1.0
    ptr, ids = torch.tensor([0, 4, 4, 12]), torch.tensor([11, 0, 5, 9, 1, 11, 11, 3, 2, 10, 8, 7], dtype=torch.int32)
    Y = csr(ptr, ids, items, gpu_device)
    want, want_states, bound, bound_states = ref.recur(ptr.numpy(), ids.numpy(), f64(V), f64(F))
    tv, tf = apart(V, gpu_device, ld), F.to(gpu_device)
    states = apart(torch.zeros((12, d), dtype=dtype), gpu_device, ld)
    last, _ = als.als_recur(ctx, Y, tv, tf, states=states)
    near(last, want, bound, F32)
    near(states, want_states, bound_states, dtype)
    ds = torch.randn((12, d), generator=torch.Generator().manual_seed(1)).to(dtype)
    dV = apart(torch.zeros((12, d), dtype=dtype), gpu_device, ld)
    dF = torch.zeros((12, d), dtype=dtype, device=gpu_device)
    als.als_recur_backward(ctx, Y, tv, tf, states, d_states=ds.to(gpu_device), out=(dV, dF, None))
    want, bound = ref.recur_backward(ptr.numpy(), ids.numpy(), f64(V), f64(F), f64(states), f64(ds))
    near(dV, want[0], bound[0], dtype)
    near(dF, want[1], bound[1], dtype)
    want, bound = ref.sum_rows(ptr.numpy(), ids.numpy(), None, f64(V))
    X = apart(torch.zeros((3, d)), gpu_device, ld)
    near(als.als_sum_rows(ctx, Y, tv, out=X), want, bound, F32)
    H = torch.randn((12, d), generator=torch.Generator().manual_seed(2))
    want, _, bound, _ = ref.recur(np.arange(13), ids.numpy(), f64(V), f64(F), f64(H)[::-1])
    X = als.als_recur_step(ctx, ids.to(gpu_device), tv, tf, apart(H, gpu_device, ld // 2), torch.arange(11, -1, -1, dtype=torch.int32, device=gpu_device))
    near(X, want, bound, F32)
    del tv, states, dV, X
    torch.cuda.empty_cache()


def test_more_entries_than_31_bits(ctx, gpu_device):
    """A short row across entry 2^31, behind one of all the entries before it (whose sum is checked against counts, to fp32's
    precision of chunks of tens of thousands of entries and their join)."""
    n, d, items = (1 << 31) + 600, 16, 1000
    say(f"als_sum_rows, als_recur: {n} entries")
    gen = torch.Generator(device=gpu_device).manual_seed(3)
    ids = torch.empty(n, dtype=torch.int32, device=gpu_device)
    counts = torch.zeros(items, dtype=torch.int64, device=gpu_device)
    first = (1 << 31) - 400
    for at in range(0, n, 1 << 28):
        part = ids[at:at + (1 << 28)]
        torch.randint(0, items, part.shape, dtype=torch.int32, device=gpu_device, generator=gen, out=part)
        counts += torch.bincount(ids[at:min(at + (1 << 28), first)].long(), minlength=items)
    E = (torch.randint(-8, 9, (items, d), generator=torch.Generator().manual_seed(1)).float() / 8).to(BF16)
    F = torch.randn((items, d), generator=torch.Generator().manual_seed(2)).to(BF16)
    ptr = torch.tensor([0, first, n])
    Y = als.Csr(2, items, ptr.to(gpu_device), ids)
    X = f64(als.als_sum_rows(ctx, Y, E.to(gpu_device)))
    tail = ids[first:].cpu().numpy()
    want, bound = ref.sum_rows(np.array([0, tail.size]), tail, None, f64(E))
    assert np.all(np.abs(X[1] - want[0]) <= bound[0])
    # the sums themselves: eighths, so every partial sum below 2^21 is exact; above, half a unit of 2^-24 relative for each of some 2^17 joins
    # of chunks, whose partial sums are a walk of steps below 1 about a drift
    drift = (f64(E) * counts.cpu().double().numpy()[:, None]).sum(0)
    assert np.all(np.abs(X[0] - drift) <= 2.0 ** 17 * 2.0 ** -24 * (np.abs(drift) + 2.0 ** 21))
    last, _ = als.als_recur(ctx, Y, E.to(gpu_device), F.to(gpu_device))
    want, _, bound, _ = ref.recur(np.array([0, tail.size]), tail, f64(E), f64(F))
    near(last[1:], want, bound, F32)
    # the long row's last state is that of its last 4000 entries: gates below 0.99 keep less than 2^-57 of what was before
    tail = ids[first - 4000:first].cpu().numpy()
    assert f64(F).max() < 4.5
    want, _, bound, _ = ref.recur(np.array([0, tail.size]), tail, f64(E), f64(F))
    near(last[:1], want, bound, F32)
    del ids, Y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("d,dtype", [(16, F32), (128, F32), (64, BF16)])
@pytest.mark.parametrize("pattern", ["stairs", "equal 64", "equal 65", "equal 512", "one long between", "alternating", "empty stretches"])
def test_rows_about_the_borders(ctx, gpu_device, d, dtype, pattern):
    """Rows that begin, end and cross at every place of chunks (multiples of 64, tiles, stages of 128 and 512) in one call."""
    if pattern == "stairs":
        lengths = list(range(0, 140)) + list(range(139, 0, -3))
    elif pattern.startswith("equal"):
        lengths = [int(pattern.split()[1])] * (8000 // int(pattern.split()[1]))
    elif pattern == "one long between":
        lengths = [1] * 63 + [2001] + [1] * 130 + [64, 128, 0, 256]
    elif pattern == "alternating":
        lengths = [300, 1, 0, 129, 1, 700] * 5
    else:
        lengths = [0] * 500 + [70] + [0] * 9000 + [1, 0, 200] + [0] * 300
    say(f"als_recur, als_recur_backward, als_sum_rows d={d} {dtype} rows {pattern}")
    items = 40
    V, F = tables(items, d, dtype, 7)
    ptr, ids = history(lengths, items, 3)
    Y = csr(ptr, ids, items, gpu_device)
    rows, n = len(lengths), ids.numel()
    gen = torch.Generator().manual_seed(4)
    H0, dl, ds = torch.randn((rows, d), generator=gen), torch.randn((rows, d), generator=gen), torch.randn((n, d), generator=gen)
    dev = [t.to(gpu_device) for t in (V, F, H0, ds, dl)]
    want, want_states, bound, bound_states = ref.recur(ptr.numpy(), ids.numpy(), f64(V), f64(F), f64(H0))
    last, states = als.als_recur(ctx, Y, *dev[:3], all_states=True)
    near(last, want, bound, F32)
    near(states, want_states, bound_states, F32)
    near(als.als_recur(ctx, Y, *dev[:3])[0], want, bound, F32)
    got = als.als_recur_backward(ctx, Y, dev[0], dev[1], states, dev[3], dev[4], dev[2])
    want, bound = ref.recur_backward(ptr.numpy(), ids.numpy(), f64(V), f64(F), f64(states), f64(ds), f64(dl), f64(H0))
    for g, w, b in zip(got, want, bound):
        near(g, w, b, F32)
    want, bound = ref.sum_rows(ptr.numpy(), ids.numpy(), None, f64(V))
    near(als.als_sum_rows(ctx, Y, dev[0]), want, bound, F32)


def test_two_recordings_share_a_workspace(gpu_device):
    """Replayed in turn, with live calls of other sizes between: the same bits as live."""
    say("als_recur, als_sum_rows, als_clip: two graphs of one context in turn")
    ctx, other = als.Context(0), als.Context(0)
    gen = torch.Generator().manual_seed(5)
    V, F = (torch.randn((50, 32), generator=gen).to(gpu_device) for _ in range(2))
    lists = [csr(*history(lengths, 50, 1), 50, gpu_device) for lengths in ([3000, 5, 0, 700], [1, 2, 20_000, 64, 64])]

    def call(c, Y):
        last, states = als.als_recur(c, Y, V, F, all_states=True)
        grads = als.als_recur_backward(c, Y, V, F, states, d_last=last)[:2]
        out = [torch.empty_like(t) for t in grads]
        return [last, states, *grads, als.als_sum_rows(c, Y, V), als.als_clip(c, grads, 0.5, out=out), *out]

    graphs, recorded = [], []
    for Y in lists:  # the first calls of the context are recorded ones
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            recorded.append(call(ctx, Y))
    for _ in range(3):
        V.add_(0.25)
        want = [call(other, Y) for Y in lists]
        for g, r, w in zip(graphs, recorded, want):
            g.replay()
            torch.cuda.synchronize()
            for a, b in zip(r, w):
                assert torch.equal(a, b)
            for a, b in zip(call(ctx, lists[0]), want[0]):
                assert torch.equal(a, b)
    ctx.close()
    other.close()


def test_clip_of_a_tensor_beyond_31_bits(ctx, gpu_device):
    n = (1 << 31) + 5
    say(f"als_clip: {n} bf16 values and 3")
    x = torch.full((n,), 0.5, dtype=BF16, device=gpu_device)
    y = torch.full((3,), 2.0, device=gpu_device)
    x[n - 1], x[n - 2] = 64.0, -8.0
    norm = (0.25 * (n - 2) + 64.0 ** 2 + 64.0 + 12.0) ** 0.5
    got = als.als_clip(ctx, [x, y], norm / 4)
    torch.cuda.synchronize()
    assert abs(float(got) - norm) <= 1e-12 * norm
    assert torch.all(x[:n - 2] == 0.125) and x[n - 2:].tolist() == [-2.0, 16.0]
    assert torch.allclose(y, torch.full_like(y, 0.5), rtol=1e-6)
    del x
    torch.cuda.empty_cache()


def test_reorder_of_rows_beyond_32_bits(ctx, gpu_device):
    cols = (1 << 30) + 7
    say(f"als_reorder: 4 rows of {cols} 16-bit values, in place and not")
    x = torch.empty((4, cols), dtype=torch.int16, device=gpu_device)
    for r in range(4):
        x[r] = r + 1
        x[r, -1] = -r - 1
    parents = torch.tensor([3, 1, 1, -1], dtype=torch.int32, device=gpu_device)
    y = torch.empty_like(x)
    als.als_reorder(ctx, parents, 4, [x], out=[y])
    als.als_reorder(ctx, parents, 4, [x])
    torch.cuda.synchronize()
    assert torch.equal(x, y)
    for r, v in enumerate((4, 2, 2, 0)):
        assert torch.all(x[r, :-1] == v) and int(x[r, -1]) == -v
    del x, y
    torch.cuda.empty_cache()


def test_many_groups_of_beams(ctx, gpu_device):
    """More groups than a grid holds workgroups, one beam each: the candidate with the best total of every row."""
    say("als_beam, als_reorder: 1.2 million groups")
    groups, k = 1_200_000, 2
    gen = torch.Generator().manual_seed(1)
    scores = torch.randint(-50, 50, (groups, k), generator=gen).float()
    ids = torch.arange(groups * k, dtype=torch.int32).view(groups, k)
    parents, items, totals, lengths = als.als_beam(ctx, ids.to(gpu_device), scores.to(gpu_device), None, torch.zeros(groups, device=gpu_device), 1)
    state = torch.arange(groups, dtype=torch.int32, device=gpu_device)
    als.als_reorder(ctx, parents, 1, [state])
    torch.cuda.synchronize()
    best = (scores[:, 1] > scores[:, 0]).long()
    assert torch.equal(items.cpu().long(), torch.arange(groups) * k + best) and torch.equal(totals.cpu(), scores.amax(1))
    assert torch.equal(parents.cpu(), torch.arange(groups, dtype=torch.int32)) and torch.all(lengths == 1)
    assert torch.equal(state.cpu(), torch.arange(groups, dtype=torch.int32))


def test_what_the_c_interface_allows(ctx, gpu_device):
    say("als_beam without lengths, als_recur without last states, als_clip of nothing, als_reorder of nothing")
    lib, dev = ctx.lib, gpu_device
    ids = torch.tensor([[4, 9], [7, 2]], dtype=torch.int32, device=dev)
    scores = torch.tensor([[3.0, 1.0], [2.5, 2.0]], device=dev)
    out = [torch.zeros(2, dtype=torch.int32, device=dev) for _ in range(2)] + [torch.zeros(2, device=dev)]
    zeros = torch.zeros(2, device=dev)
    b = als.c_als_beams(1, 2, 2, ids.data_ptr(), scores.data_ptr(), None, zeros.data_ptr(), None, None, None, 0, 0, 1.0)
    assert lib.als_beam(ctx.handle, ctypes.byref(b), out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(), None, None) == als.ALS_OK
    torch.cuda.synchronize()
    assert [t.tolist() for t in out] == [[0, 1], [4, 7], [3.0, 2.5]]
    V, F = torch.randn((6, 16), device=dev), torch.randn((6, 16), device=dev)
    Y = als.Csr(2, 6, torch.tensor([0, 2, 3], device=dev), torch.tensor([5, 0, 1], dtype=torch.int32, device=dev))
    states = torch.zeros((3, 16), device=dev)
    y, tv, tf, ts = Y.c(), als._table(V), als._table(F), als._table(states)
    assert lib.als_recur(ctx.handle, ctypes.byref(y), ctypes.byref(tv), ctypes.byref(tf), None, ctypes.byref(ts), None, None) == als.ALS_OK
    _, want = als.als_recur(ctx, Y, V, F, all_states=True)
    torch.cuda.synchronize()
    assert torch.equal(states, want)
    assert float(als.als_clip(ctx, [], 1.0)) == 0.0
    assert float(als.als_clip(ctx, [torch.zeros((0, 5), device=dev), torch.zeros(0, dtype=BF16, device=dev)], 1.0)) == 0.0
    assert als.als_reorder(ctx, torch.zeros(0, dtype=torch.int32, device=dev), 4, [torch.zeros((0, 3), device=dev)])[0].shape == (0, 3)
    als.als_reorder(ctx, torch.zeros(2, dtype=torch.int32, device=dev), 2, [])
    got = als.als_beam(ctx, ids[:0], scores[:0], None, None, 3)
    assert [t.numel() for t in got] == [0, 0, 0, 0]
    torch.cuda.synchronize()


def the_example():
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "next_items.py")
    spec = importlib.util.spec_from_file_location("next_items", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_the_example_continues_histories(gpu_device):
    say("examples/next_items.py")
    r = the_example().main(nodes=6000, epochs=2, gate_steps=3, answered=20)
    assert all(np.isfinite(v) for pair in r["training"] for v in pair) and 0 < r["gates"] < 1
    items, total = r["items"], r["log_probability"]
    assert items.shape == (20, 4, 5) and torch.all(items >= 0)
    for row in items.view(-1, 5).tolist():
        assert len(set(row)) == 5  # no item twice
    assert torch.all(total <= 1e-4) and torch.all(total[:, :-1] >= total[:, 1:])


def test_the_gradients_of_the_example_are_differences(ctx, gpu_device):
    """Directions in the tables that the recurrence reads, with the items that queries are compared with held.  The loss in 64 bits by
    the reference; central differences with a step of 2^-12 are off by 2^-24 / 6 of third derivatives, the gradients by some
    hundred fp32 roundings: below 1e-4 of the sum of the magnitudes that go into the product."""
    say("examples/next_items.py: gradients against differences")
    ex = the_example()
    gen = torch.Generator().manual_seed(2)
    items, d = 30, 16
    V, F = (torch.randn((items, d), generator=gen).to(gpu_device) for _ in range(2))
    Y = csr(*history([4, 0, 9, 130, 1, 2], items, 3, stray=False), items, gpu_device)
    by_item = ex.entries_by_item(Y.indices, items)
    _, gV, gF = ex.loss_and_gradients(ctx, Y, by_item, V, F)
    behind, some = ex.next_entries(Y.indptr, Y.nnz)
    target = V[Y.indices[behind].long()].double()

    def loss(v, f):
        states = torch.from_numpy(ref.recur(Y.indptr.cpu().numpy(), Y.indices.cpu().numpy(), f64(v), f64(f))[1]).to(gpu_device)
        return float(torch.where(some[:, None], states - target, 0.0).square().sum() / (2 * some.sum()))

    for k, grad in enumerate((gV, gF)):
        for _ in range(2):
            way = torch.randn((items, d), generator=gen).to(gpu_device)
            step = 2.0 ** -12
            up, down = (loss(V.double() + (s * step * way.double() if k == 0 else 0), F.double() + (s * step * way.double() if k == 1 else 0)) for s in (1, -1))
            want = (up - down) / (2 * step)
            assert abs(float((grad.double() * way.double()).sum()) - want) <= 1e-4 * float((grad.double() * way.double()).abs().sum()) + 1e-9


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape,gap", [((3000, 1), 2), ((1025, 16), 16), ((777, 65), 7), ((2049, 128), 1), ((33, 4095), 5), ((5, 4097), 9),
                                       ((1, 9), 1), ((2, 2), 1000)])
def test_clip_of_rows_with_gaps(ctx, gpu_device, shape, gap, dtype):
    """Several rows share a tile where they are short; what lies between rows is neither counted nor written."""
    say(f"als_clip: {shape} with gaps of {gap}, {dtype}")
    gen = torch.Generator().manual_seed(5)
    host = torch.randn(shape, generator=gen).to(dtype)
    other = torch.randn(100, generator=gen).to(dtype)

    def with_gaps(fill):
        big = torch.full((shape[0], shape[1] + gap), fill, dtype=dtype, device=gpu_device)
        return big, big[:, :shape[1]]

    norm = torch.sqrt(wide(host).square().sum() + wide(other).square().sum()).item()
    bound = norm / 3
    for place in ("in place", "out"):
        big, x = with_gaps(1e30)
        x.copy_(host.to(gpu_device))
        lone = other.to(gpu_device)
        out = None
        if place == "out":
            far, y = with_gaps(-7.0)
            out = [y, torch.empty_like(lone)]
        got = als.als_clip(ctx, [x, lone], bound, out=out)
        assert abs(got.item() - norm) <= (host.numel() + other.numel() + 4) * 2.0 ** -53 * norm  # as many additions in fp64
        space, written = (far, y) if out else (big, x)
        assert torch.all(space[:, shape[1]:] == (torch.tensor(-7.0) if out else torch.tensor(1e30)).to(dtype).to(gpu_device))
        # the factor, the product and the stored value are rounded once each
        want = wide(host) * (bound / norm)
        tol = 2 * 2.0 ** -24 + torch.finfo(dtype).eps / 2
        assert torch.all((wide(written) - want).abs() <= 1.01 * tol * want.abs() + 1e-38)
        if out:
            assert torch.equal(x.cpu(), host)
