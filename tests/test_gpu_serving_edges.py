"""Answering from trained tables on the GPU where it is easy to go wrong: scores far from zero, shapes that reach the inner loops
of every kernel, recordings beside live calls of another size.

References are plain 64-bit computations (serving_ref on the CPU; for large shapes elementary torch operations in 64 bits on the
GPU).  Bounds stand at each test, derived before any run.
"""
import numpy as np
import pytest
import torch

import serving_ref as ref
from gpu_util import f64, rel_fro, say
from paper_2112_02194_amd import binding as als
from synth import init_table, make_problem
from test_gpu_serving import check_selected, to_ref, to_rules

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(gpu_device):
    c = als.Context(0)
    yield c
    c.close()


# ------------------------------------------------------------------------------------------------ log-sum-exp

def far_rows(n, kind, gen):
    """Rows of finite scores, all or some of them far from zero."""
    x = torch.randn((4, n), generator=gen)
    if kind == "ordinary":
        return x
    if kind.startswith("stretch"):  # a finite number where others would put -inf, in whole stretches, in most places, in all but one
        value = -float(kind.split()[1])
        x[0, : n // 2] = value
        x[1, n // 3:] = value
        x[2, torch.rand(n, generator=gen) < 0.9] = value
        x[3, 1:] = value
        return x
    size = float(kind)  # scores about that large, a few steps apart: the largest counts, or some of them
    return torch.tensor(size) * (1 + 2.0 ** -20 * torch.randint(-3, 4, (4, n), generator=gen)) + x


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind,temperature", [
    ("1e5", 1.0), ("3e6", 1.0), ("-3e6", 1.0), ("2e9", 1.0), ("1e10", 1.0), ("1.1e10", 1.0), ("-1e10", 1.0), ("1e12", 1.0), ("1e20", 1.0),
    ("-1e20", 1.0), ("1e30", 3.0), ("ordinary", 1e-10), ("ordinary", 1e-6), ("ordinary", 1e30), ("stretch 1e6", 1.0), ("stretch 1e9", 0.1),
    ("stretch 1e10", 1.0), ("stretch 1e20", 1.0), ("stretch 3e38", 1.0), ("1e7", 1e7)])
def test_lse_of_scores_far_from_zero(ctx, gpu_device, kind, temperature, dtype):
    """Bounds: check_selected's, whose terms grow with the scores."""
    t = float(np.float32(temperature))
    for n in (1, 3, 700, 5000, 70_001):
        say(f"als_select 4 x {n}, scores {kind}, temperature {temperature} {dtype}")
        x = far_rows(n, kind, torch.Generator().manual_seed(n)).to(dtype)
        got = als.als_select(ctx, x.to(gpu_device), 3, temperature=temperature)
        torch.cuda.synchronize()
        check_selected(got, f64(x), 3, t, n)


def test_lse_of_biases_and_histories_far_from_zero(ctx, gpu_device):
    say("als_select 3 x 9000, half the items by a bias of -1e10, penalties of 1e12")
    gen = torch.Generator().manual_seed(1)
    n = 9000
    x = (torch.randn((3, n), generator=gen) * 8).round() / 8
    bias = torch.where(torch.rand(n, generator=gen) < 0.5, -1e10, 0.0)
    bias[: n // 3] = -1e10
    indptr = torch.tensor([0, 300, 300, 320])
    ids = torch.randint(0, n, (320,), generator=gen).to(torch.int32)
    history = als.Csr(3, n, indptr.to(gpu_device), ids.to(gpu_device))
    got = als.als_select(ctx, x.to(gpu_device), 5, als.Rules(history=history, presence=1e12, bias=bias.to(gpu_device)))
    torch.cuda.synchronize()
    want, _ = ref.adjust(f64(x), history=(indptr.numpy(), ids.numpy()), presence=float(np.float32(1e12)), bias=bias.numpy())
    _, _, lse = ref.select(want, 5)
    top = np.abs(want.max(1))
    bound = (np.log2(n + 1) + 4) * 2.0 ** -22 + 2.0 ** -22 * (np.abs(lse) + 2 * top)
    assert np.all(np.abs(f64(got[2]) - lse) <= bound)


@pytest.mark.parametrize("temperature", [3.0, 0.3, 0.037, 0.01, 0.0013, 0.0001])
def test_lse_is_as_exact_as_its_largest_part(ctx, gpu_device, temperature):
    """lse = m / t + log(sum): one rounding each of the quotient and of the last sum, halves of a unit of |m / t| and |lse|, and the
    sum's relative error in units of 2^-24: exponents of the terms, from three roundings of numbers whose mean, weighted by the terms,
    is at most log2(n), in the terms and again where sums of lanes are joined (3.5 log2(n)); exponentials and their joining of
    two units (8); at most 20 additions one after the other; the logarithm itself (2 |log sum|)."""
    n, rows = 1000, 64
    say(f"als_select {rows} x {n}, temperature {temperature}: distance of lse")
    t = float(np.float32(temperature))
    x = torch.randn((rows, n), generator=torch.Generator().manual_seed(7)) * 1.5
    for scale in (1.0, 1.07, 1.23, 1.37, 1.71, 1.93):
        y = x * scale
        _, _, lse = als.als_select(ctx, y.to(gpu_device), 1, temperature=temperature)
        torch.cuda.synchronize()
        _, _, want = ref.select(f64(y), 1, t)
        m = f64(y).max(1) / t
        bound = 2.0 ** -24 * (np.abs(m) + np.abs(want) + 2 * np.abs(want - m) + 3.5 * np.log2(n) + 28)
        assert np.all(np.abs(f64(lse) - want) <= bound)


# ------------------------------------------------------------------------------------------------ recordings

def test_a_recorded_selection_beside_larger_live_ones(gpu_device):
    """The workspace of a recording must be the one it was recorded with, whatever is called on the context between its replays: calls
    with many more parts of rows, of another kernel, for other rows.  The recorded call is the context's first."""
    say("als_select: recorded as a context's first call, replayed between larger live calls")
    gen = torch.Generator().manual_seed(11)
    X = torch.randn((2, 50_001), generator=gen).to(gpu_device)
    large = [torch.randn(shape, generator=gen).to(gpu_device) for shape in ((1, 3_000_001), (64, 300_000), (300, 30_000), (1500, 9000))]
    ctx, other = als.Context(0), als.Context(0)
    want = [als.als_select(other, t, 20, temperature=0.8) for t in large]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        recorded = als.als_select(ctx, X, 20, temperature=0.8)
    for t, w in zip(large, want):
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(als.als_select(ctx, t, 20, temperature=0.8), w):
            assert torch.equal(a, b)
        X.copy_(torch.randn(X.shape, generator=gen))
        for a in recorded:
            a.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(recorded, als.als_select(other, X, 20, temperature=0.8)):
            assert torch.equal(a, b)
    ctx.close()
    other.close()


def test_selection_allocates_nothing(gpu_device):
    say("als_select: free memory of the card before and after calls of growing size")
    ctx = als.Context(0)
    X = torch.randn((512, 200_000), generator=torch.Generator().manual_seed(1)).to(gpu_device)
    als.als_select(ctx, X[:1, :100], 5)
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    for rows, cols in ((1, 5000), (1, 200_000), (8, 200_000), (64, 200_000), (512, 200_000)):
        als.als_select(ctx, X[:rows, :cols], 5)
        torch.cuda.synchronize()
    assert free - torch.cuda.mem_get_info()[0] < 1 << 20  # torch's own results fit a block that it has; the old workspace was 10 MB
    ctx.close()


def test_recordings_of_growing_calls_beside_larger_live_ones(gpu_device):
    """als_gramian, als_solve_rows, als_topk and als_epoch grow their workspace on demand: a recording keeps the buffers that it holds."""
    say("als_epoch, als_solve_rows, als_topk: replayed between larger live calls")
    small, large = make_problem("c1", rows=700, cols=600), make_problem("c1", rows=40_000, cols=30_000)
    dev, prm = gpu_device, als.make_params(small.alpha, small.lam)
    ctx, other = als.Context(0), als.Context(0)

    def held(p):
        Y = als.Csr(p.rows, p.cols, p.indptr.to(dev), p.indices.to(dev))
        Yt = als.Csr(p.cols, p.rows, p.t_indptr.to(dev), p.t_indices.to(dev))
        return Y, Yt, p.W0.to(dev), p.H0.to(dev), torch.zeros_like(p.W0, device=dev)

    def step(c, Y, Yt, W, H, X):
        als.als_epoch(c, Y, Yt, W, H, prm)
        als.als_solve_rows(c, Y, H, als.als_gramian(c, H), prm, X)
        return als.als_topk(c, X, H, 10)

    S, L, S2, L2 = held(small), held(large), held(small), held(large)
    step(ctx, *S)  # the workspace takes this problem's size
    als.als_status_sync(ctx)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ids, scores = step(ctx, *S)
    torch.cuda.synchronize()
    for _ in range(3):
        got = step(ctx, *L)  # outgrows it, the first time
        want = step(other, *L2)
        torch.cuda.synchronize()
        assert rel_fro(f64(L[2]), f64(L2[2])) <= 1e-6 and torch.allclose(got[1], want[1], rtol=1e-4, atol=1e-6)
        for t, p in ((S, small), (S2, small)):
            t[2].copy_(p.W0)
            t[3].copy_(p.H0)
        ids.zero_()
        torch.cuda.synchronize()
        graph.replay()
        want = step(other, *S2)
        torch.cuda.synchronize()
        assert rel_fro(f64(S[2]), f64(S2[2])) <= 1e-6 and rel_fro(f64(S[3]), f64(S2[3])) <= 1e-6  # grids may differ from live calls
        assert rel_fro(f64(S[4]), f64(S2[4])) <= 1e-6 and torch.allclose(scores, want[1], rtol=1e-4, atol=1e-6)
        again = als.als_topk(other, S[4], S[3], 10)
        torch.cuda.synchronize()
        assert torch.equal(ids, again[0]) and torch.equal(scores, again[1])
    ctx.close()
    other.close()


# ------------------------------------------------------------------------------------------------ scores

def scores_bound(Q, V, d, want, ds):
    """d fp32 products and their sum in any order, an entry rounded to at least 19 bits (2^-19 = 32 units of 2^-24 where entries are
    far apart, 4 units elsewhere), a scale: (2 d + 16) 2^-24 sum_j |q_j v_ij| holds for both with d >= 16, since the sum's
    d units are met by d - 1 additions at most; half an ulp of a bf16 result."""
    bound = (2 * d + 16) * 2.0 ** -24 * (np.abs(Q) @ np.abs(V).T) + 1e-37
    return bound if ds == torch.float32 else bound * (1 + 2.0 ** -7) + np.abs(want) * 2.0 ** -8


PAIRS = [(16, 16), (32, 16), (32, 32), (64, 16), (64, 32), (64, 64), (128, 16), (128, 32), (128, 64), (128, 128)]


@pytest.mark.parametrize("dq", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d,group", PAIRS)
def test_scores_of_queries_with_entries_far_apart(ctx, gpu_device, d, group, dq):
    """One large entry in a query's row, in an item whose code there is 0: the score is made of the small ones alone, and has their
    bits, however many queries there are in the call."""
    gen = torch.Generator().manual_seed(d + group)
    n = 700
    X = torch.randn((n, d), generator=gen)
    X[: n // 2, d // 3] = 0.0
    X[n // 2: n // 2 + 9, d // 3 + 1:] = 0.0  # others at the large entry alone, or mixed
    T = als.als_quantize(ctx, X.to(gpu_device), group)
    V = f64(als.als_dequantize(ctx, T))
    for nq in (1, 2, 4, 5, 31, 40, 70):
        for power in (-10, -16, -19, -20, -21, -30, -33, -40, -60, -100):
            say(f"als_scores nq={nq} d={d} group={group} {dq}: entries 2^{power} of the largest")
            Q = torch.randn((nq, d), generator=gen)
            Q = torch.where(Q.abs() < 0.25, torch.full_like(Q, 0.25), Q) * 2.0 ** power
            Q[::3, d // 3] = 5.0  # the other rows are ordinary ones
            if nq > 31:
                Q[3] *= 1e20  # and one is far from 1
            Q = Q.to(dq)
            for ds, pad in ((torch.float32, 0), (torch.bfloat16, 1)):
                big = torch.full((nq + 1, n + pad), 9.0, dtype=ds, device=gpu_device)
                als.als_scores(ctx, Q.to(gpu_device), T, out=big[:nq, :n])
                torch.cuda.synchronize()
                want = f64(Q) @ V.T
                assert np.all(np.abs(f64(big[:nq, :n]) - want) <= scores_bound(f64(Q), V, d, want, ds))
                assert torch.all(big[nq:] == 9.0) and torch.all(big[:, n:] == 9.0)


@pytest.mark.parametrize("nq", [1, 5, 40])
def test_scores_of_infinite_entries_beside_small_ones(ctx, gpu_device, nq):
    say(f"als_scores: infinite and NaN entries in rows with entries far apart, nq={nq}")
    d, n = 64, 300
    gen = torch.Generator().manual_seed(3)
    T = als.als_quantize(ctx, torch.randn((n, d), generator=gen).to(gpu_device), 32)
    V = f64(als.als_dequantize(ctx, T))
    Q = torch.randn((nq, d), generator=gen)
    Q[:, 7] *= 2.0 ** -60
    plain = f64(als.als_scores(ctx, Q.to(gpu_device), T))
    Q[0, 5] = float("inf")
    S = f64(als.als_scores(ctx, Q.to(gpu_device), T))
    with np.errstate(all="ignore"):
        assert np.array_equal(S[0], np.where(V[:, 5] == 0, np.nan, np.inf * V[:, 5]), equal_nan=True)
    assert np.array_equal(S[1:], plain[1:])
    Q[0, 5] = float("nan")
    S = f64(als.als_scores(ctx, Q.to(gpu_device), T))
    assert np.all(np.isnan(S[0])) and np.array_equal(S[1:], plain[1:])


@pytest.mark.parametrize("nq", [1, 2, 3, 4, 40])
@pytest.mark.parametrize("dq", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("big,small", [(-124, 100), (-126, 124), (-132, 120), (-16, 120), (-15, 110), (-60, 124)])
def test_scores_of_queries_near_the_end_of_the_range(ctx, gpu_device, nq, dq, big, small):
    """Entries at and below the smallest normal number keep the bits that they have: what a query is scaled by may not take them."""
    say(f"als_scores: queries times 2^{big}, tables times 2^{small}, nq={nq} {dq}")
    for d, group in ((16, 16), (32, 32), (64, 32), (128, 128)):
        T = als.als_quantize(ctx, (init_table(300, d, seed=4, stream=1).clamp(-3, 3) * 2.0 ** small).to(gpu_device), group)
        Q = (init_table(nq, d, seed=6, stream=2).clamp(-1, 1) * 2.0 ** big).to(dq)
        S = f64(als.als_scores(ctx, Q.to(gpu_device), T))
        V, Qh = f64(als.als_dequantize(ctx, T)), f64(Q)
        assert np.all(np.isfinite(V))
        want = Qh @ V.T
        assert np.all(np.abs(S - want) <= scores_bound(Qh, V, d, want, torch.float32))


# ------------------------------------------------------------------------------------------------ shapes that reach the inner loops

def close_on_gpu(S, Q, T, ctx, ds):
    """scores_bound on the GPU, a million items at a time."""
    d, Qd = Q.shape[1], Q.double()
    for i in range(0, S.shape[1], 1 << 20):
        part = als.QTable(T.codes[i:i + (1 << 20)], T.scales[i:i + (1 << 20)])
        Vt = als.als_dequantize(ctx, part).double().T.contiguous()
        want = Qd @ Vt
        bound = (2 * d + 16) * 2.0 ** -24 * (Qd.abs() @ Vt.abs()) + 1e-37
        if ds == torch.bfloat16:
            bound = bound * (1 + 2.0 ** -7) + want.abs() * 2.0 ** -8
        if not bool(((S[:, i:i + (1 << 20)].double() - want).abs() <= bound).all()):
            return False
    return True


def random_table(n, d, group, gen, dev):
    codes = torch.randint(0, 256, (n, d // 2), dtype=torch.uint8, device=dev, generator=gen)
    return als.QTable(codes, (0.02 * torch.rand((n, d // group), device=dev, generator=gen) + 0.001).to(torch.bfloat16))


@pytest.mark.parametrize("dq", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("ds", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d,group", PAIRS)
def test_scores_over_several_rounds(ctx, gpu_device, d, group, dq, ds):
    """500 queries against enough items that a wavefront walks six rounds (rows of whole 128-byte lines) or two (rows that share
    lines; bf16 rows of odd length take the form without a bounds check), the last ones not whole."""
    gen = torch.Generator(device=gpu_device).manual_seed(d + group)
    for n, ld in ((98_560, 98_560), (98_501, 98_560), (98_501, 98_501), (98_502, 98_502)):
        say(f"als_scores 500 x {n} (rows of {ld}) d={d} group={group} {dq} -> {ds}")
        T = random_table(n, d, group, gen, gpu_device)
        Q = torch.randn((500, d), device=gpu_device, generator=gen)
        Q = torch.where(Q.abs() < 1e-4, torch.full_like(Q, 1e-4), Q).to(dq)
        if n != 98_560:
            Q[65, 3] = 1e-12  # one group of queries in the form for entries far apart
        big = torch.full((501, ld), 9.0, dtype=ds, device=gpu_device)
        als.als_scores(ctx, Q, T, out=big[:500, :n])
        torch.cuda.synchronize()
        assert close_on_gpu(big[:500, :n], Q, T, ctx, ds)
        assert bool((big[500] == 9.0).all()) and bool((big[:500, n:] == 9.0).all())
        del big


@pytest.mark.parametrize("ds", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d,group,n", [(16, 16, 4_500_001), (32, 16, 4_500_001), (32, 32, 4_500_001), (64, 16, 2_300_003), (64, 64, 2_300_003),
                                       (128, 16, 1_300_007), (128, 32, 1_300_007), (128, 128, 1_300_007)])
def test_scores_of_few_queries_over_several_rounds(ctx, gpu_device, d, group, n, ds):
    gen = torch.Generator(device=gpu_device).manual_seed(d + group)
    T = random_table(n, d, group, gen, gpu_device)
    for nq, dq in ((1, torch.float32), (2, torch.bfloat16), (3, torch.float32), (4, torch.float32), (4, torch.bfloat16)):
        say(f"als_scores {nq} x {n} d={d} group={group} {dq} -> {ds}")
        Q = torch.randn((nq, d), device=gpu_device, generator=gen).to(dq)
        S = als.als_scores(ctx, Q, T, dtype=ds)
        torch.cuda.synchronize()
        assert close_on_gpu(S, Q, T, ctx, ds)


@pytest.mark.parametrize("rows,d,group,dtype", [(600_001, 128, 32, torch.float32), (1_100_003, 128, 128, torch.bfloat16), (4_300_001, 16, 16, torch.float32)])
def test_quantize_of_more_rows_than_a_grid_takes_at_once(ctx, gpu_device, rows, d, group, dtype):
    """Parts of the table, each of one turn of the grid, have the same bits as the whole, and some rows at every turn's ends those of
    the definition."""
    say(f"als_quantize, als_dequantize {rows} x {d} groups of {group} {dtype}")
    gen = torch.Generator(device=gpu_device).manual_seed(5)
    X = (torch.randn((rows, d), device=gpu_device, generator=gen) * torch.exp(torch.randn((rows, 1), device=gpu_device, generator=gen))).to(dtype)
    T = als.als_quantize(ctx, X, group)
    back = als.als_dequantize(ctx, T)
    half = als.als_dequantize(ctx, T, dtype=torch.bfloat16)
    torch.cuda.synchronize()
    turn = 16_384 * 1024 // (d // (4 if dtype == torch.float32 else 8))
    step = turn // 2 + 3
    for i in range(0, rows, step):
        P = als.als_quantize(ctx, X[i:i + step], group)
        assert torch.equal(P.codes, T.codes[i:i + step]) and torch.equal(P.scales, T.scales[i:i + step])
        assert torch.equal(als.als_dequantize(ctx, P), back[i:i + step])
        assert torch.equal(als.als_dequantize(ctx, P, dtype=torch.bfloat16), half[i:i + step])
    for i in (0, turn - 700, rows - 700):
        code, scale = ref.quantize(X[i:i + 700].float().cpu().numpy(), group)
        assert np.array_equal(T.codes[i:i + 700].cpu().numpy(), ref.pack(code))
        assert np.array_equal(f64(T.scales[i:i + 700]), scale.astype(np.float64))
        assert np.array_equal(f64(back[i:i + 700]), ref.values(code, scale))


def lists_of_lengths(rows, cols, lengths, gen, values):
    n = torch.tensor([lengths[q % len(lengths)] for q in range(rows)])
    indptr = torch.zeros(rows + 1, dtype=torch.int64)
    indptr[1:] = torch.cumsum(n, 0)
    total = int(indptr[-1])
    ids = (torch.rand(total, generator=gen) ** 2 * cols).to(torch.int32)
    return indptr, ids, (torch.randn(total, generator=gen) * 8).round() / 8 if values else None


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,k", [(128, 30_000, 20), (256, 60_000, 64), (200, 33_001, 1)])
def test_select_by_one_large_workgroup_per_row_with_every_rule(ctx, gpu_device, rows, cols, k, dtype):
    """Rows that take several tiles of the kernel with 1024 threads, lists that a wavefront holds and lists that are walked, of both
    kinds in every combination; the rules' arithmetic is exact, so ids and scores have to be equal."""
    say(f"als_select {rows} x {cols} every rule, k={k} {dtype}")
    gen = torch.Generator().manual_seed(rows)
    X = ((torch.randn((rows, cols), generator=gen) * 24).round() / 8).to(dtype)
    kw = dict(history=lists_of_lengths(rows, cols, (0, 3, 255, 256, 257, 900, 5000), gen, False), penalties=torch.tensor([[2.0, 0.5, 0.25], [0.5, 0.0, 0.125]])[torch.arange(rows) % 2],
              entries=lists_of_lengths(rows, cols, (700, 0, 257, 20, 256), gen, True), bias=(torch.randn(cols, generator=gen) * 8).round() / 8,
              allowed=torch.randint(-2 ** 31, 2 ** 31, (rows, (cols + 31) // 32), generator=gen).to(torch.int32))
    kw["allowed"][rows // 2] = 0
    kw["allowed"][3, : cols // 32 - 3] = 0  # the last items alone
    want, _ = ref.adjust(f64(X), **to_ref(kw))
    got = als.als_select(ctx, X.to(gpu_device), k, to_rules(kw, rows, cols, gpu_device), 0.5)
    torch.cuda.synchronize()
    check_selected(got, want, k, 0.5, cols)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(4, 20_011), (256, 60_000), (600, 40_001)])
def test_select_by_every_kernel_whatever_the_order(ctx, gpu_device, rows, cols, dtype):
    """Ascending, descending and equal scores, one row of each kind after the other, with histories and without: more candidates than
    a tile's buffer holds, cut back between its steps."""
    gen = torch.Generator().manual_seed(cols)
    base = torch.arange(cols, dtype=torch.float32)
    kinds = [base / 8, -base, torch.full((cols,), 2.0), base % 97, -(base // 4096)]
    X = torch.stack([kinds[q % 5] for q in range(rows)]).to(dtype)
    history = lists_of_lengths(rows, cols, (0, 3, 255, 300), gen, False)
    kw = dict(history=history, repetition=2.0, presence=0.25, frequency=0.125)
    some = sorted({0, 1, 2, 3, 4, rows // 2, rows - 1} & set(range(rows)))  # rows that are checked one by one
    cut = (torch.cat([torch.zeros(1, dtype=torch.int64), torch.cumsum(torch.tensor([int(history[0][q + 1] - history[0][q]) for q in some]), 0)]),
           torch.cat([history[1][history[0][q]:history[0][q + 1]] for q in some]), None)
    for k in (1, 64):
        say(f"als_select {rows} x {cols} ordered and equal scores, k={k} {dtype}")
        plain = als.als_select(ctx, X.to(gpu_device), k)
        ruled = als.als_select(ctx, X.to(gpu_device), k, to_rules(kw, rows, cols, gpu_device))
        torch.cuda.synchronize()
        check_selected([t[some] for t in plain], f64(X[some]), k, 1.0, cols)
        want, _ = ref.adjust(f64(X[some]), **to_ref({**kw, "history": cut}))
        # bf16 scores with a quarter or an eighth taken off are exact in fp32, so are fp32 ones up to 60 000 / 8
        check_selected([t[some] for t in ruled], want, k, 1.0, cols)
        for kind in range(min(5, rows)):  # without rules all rows of a kind have one answer
            for t in plain:
                assert bool((t[kind::5] == t[kind]).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_select_of_one_long_row_with_equal_and_ordered_scores(ctx, gpu_device, dtype):
    """Hundreds of parts that all reach the best score: more candidates than the merge holds at a time."""
    n = 3_000_001
    base = torch.arange(n, dtype=torch.float32)
    for name, x in (("equal", torch.zeros(n)), ("ascending", base / 8), ("descending", -base), ("few values", base % 3)):
        x = x.to(dtype)[None, :]
        for k in (1, 64):
            say(f"als_select 1 x {n}, {name}, k={k} {dtype}")
            got = als.als_select(ctx, x.to(gpu_device), k, temperature=4.0)
            torch.cuda.synchronize()
            check_selected(got, f64(x), k, 4.0, n)
