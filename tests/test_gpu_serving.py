"""Answering from trained tables on the GPU: 4-bit tables, scores against them, rules on scores, selection.

References are plain 64-bit computations on the CPU (serving_ref).  Bounds, before any run:
quantize, dequantize   none: the definition is a fixed sequence of IEEE operations, so codes, scales and values have its bits
scores                 the sum of d fp32 products in any order, each with a rounding of the query to at least 22 bits and of a
                       scale: (2 d + 16) 2^-24 sum_j |q_j v_ij|, plus half an ulp of a bf16 result
adjust                 at most six fp32 roundings, each of a number no larger than the magnitudes that went in: 6 * 2^-24 of
                       their sum, plus half an ulp of a bf16 result
select                 none on ids and scores where the rules' arithmetic is exact; the log-sum-exp has exponents rounded to
                       fp32 (weighted by their own exponential at most log2(n) + 4 units of 2^-22) and two sums
"""
import numpy as np
import pytest
import torch

import serving_ref as ref
from gpu_util import f64, say
from paper_2112_02194_amd import binding as als
from synth import init_table

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(gpu_device):
    c = als.Context(0)
    yield c
    c.close()


def host(t):
    return t.detach().cpu().numpy()


# ------------------------------------------------------------------------------------------------ 4-bit tables

def table(n, d, dtype, seed, special=True):
    x = init_table(n, d, seed=seed, stream=3) * torch.exp(torch.randn((n, 1), generator=torch.Generator().manual_seed(seed)))
    if special and n > 40:
        x[3] = 0.0
        x[4] = 1e-41           # below the normal range
        x[5, ::2] = -3e38
        x[6] = x[6].abs().max() * (torch.arange(d) % 15 - 7) / 7.0 * 0.5  # quotients on and near halves
        x[7, 0] = 1e-45        # a scale that rounds to zero
        x[7, 1:] = 0.0
        x[8, 1] = float("inf")
        x[9, 2] = float("nan")
        x[10, d - 1] = float("-inf")
    return x.to(dtype)


def strided(t, dev, pad):
    """The same values in a matrix whose rows are further apart, the rest filled with NaN."""
    big = torch.full((t.shape[0] + 1, t.shape[1] + pad), float("nan"), dtype=t.dtype, device=dev)
    big[:t.shape[0], :t.shape[1]] = t.to(dev)
    return big[:t.shape[0], :t.shape[1]]


@pytest.mark.parametrize("d,group", [(16, 16), (32, 16), (32, 32), (64, 16), (64, 64), (128, 16), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantize_has_the_bits_of_its_definition(ctx, gpu_device, d, group, dtype):
    for n, pad in ((1, 0), (45, 16), (1037, 0), (4099, 32)):
        say(f"als_quantize n={n} d={d} group={group} {dtype} pad={pad}")
        x = table(n, d, dtype, seed=n)
        T = als.als_quantize(ctx, strided(x, gpu_device, pad) if pad else x.to(gpu_device), group)
        back = {t: als.als_dequantize(ctx, T, dtype=t) for t in (torch.float32, torch.bfloat16)}
        wide = torch.full((n, d + 8), 5.0, device=gpu_device)
        als.als_dequantize(ctx, T, out=wide[:, :d])
        torch.cuda.synchronize()
        code, scale = ref.quantize(x.float().numpy(), group)
        assert np.array_equal(host(T.codes), ref.pack(code))
        assert np.array_equal(f64(T.scales), scale.astype(np.float64), equal_nan=True)
        v = ref.values(code, scale)
        assert np.array_equal(f64(back[torch.float32]), v, equal_nan=True)
        assert np.array_equal(f64(back[torch.bfloat16]), ref.bf16(v).astype(np.float64), equal_nan=True)
        assert np.array_equal(f64(wide[:, :d]), v, equal_nan=True) and torch.all(wide[:, d:] == 5.0)


def test_quantize_error_is_half_a_step(ctx, gpu_device):
    say("als_quantize: distance of values from the table")
    x = init_table(3001, 128, seed=2, stream=1)
    T = als.als_quantize(ctx, x.to(gpu_device), 32)
    v = f64(als.als_dequantize(ctx, T))
    s = np.repeat(f64(T.scales), 32, axis=1)
    # half a step where the code is not clipped; a scale rounded down by up to 2^-9 clips the largest by 7 * 2^-9 of a step
    assert np.all(np.abs(v - f64(x)) <= s * (0.5 + 1e-6))


@pytest.mark.parametrize("dq", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("ds", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d,group", [(16, 16), (32, 16), (32, 32), (64, 32), (64, 64), (128, 16), (128, 32), (128, 128)])
def test_scores_match_the_definition(ctx, gpu_device, d, group, dq, ds):
    for nq, n, pad in ((1, 1, 0), (1, 4099, 0), (2, 777, 3), (3, 64, 1), (5, 257, 0), (32, 31, 0), (33, 1025, 2), (70, 2113, 0), (257, 515, 1)):
        say(f"als_scores nq={nq} n={n} d={d} group={group} {dq} -> {ds} pad={pad}")
        T = als.als_quantize(ctx, table(n, d, torch.float32, seed=n + d, special=False).to(gpu_device), group)
        Q = init_table(nq, d, seed=nq, stream=5) * 10
        Q[nq // 2, : d // 2] *= 1e-6   # entries of very different size in one row
        if nq > 2:
            Q[1] = 0.0
            Q[2] *= 1e30
        Q = Q.to(dq)
        Sbig = torch.full((nq + 1, n + pad), 9.0, dtype=ds, device=gpu_device)
        S = Sbig[:nq, :n]
        als.als_scores(ctx, strided(Q, gpu_device, 16) if pad else Q.to(gpu_device), T, out=S)
        torch.cuda.synchronize()
        V, Qh = f64(als.als_dequantize(ctx, T)), f64(Q)
        want, bound = Qh @ V.T, (2 * d + 16) * 2.0 ** -24 * (np.abs(Qh) @ np.abs(V).T) + 1e-37
        if ds == torch.bfloat16:
            bound = bound * (1 + 2.0 ** -7) + np.abs(want) * 2.0 ** -8
        assert np.all(np.abs(f64(S) - want) <= bound)
        assert torch.all(Sbig[nq:] == 9.0) and torch.all(Sbig[:, n:] == 9.0)


@pytest.mark.parametrize("nq", [1, 2, 40])
def test_scores_of_values_that_are_not_finite(ctx, gpu_device, nq):
    say(f"als_scores: infinite and NaN scales and queries, nq={nq}")
    x = table(300, 64, torch.float32, seed=5)
    T = als.als_quantize(ctx, x.to(gpu_device), 32)
    Q = init_table(nq, 64, seed=3, stream=2)
    S = f64(als.als_scores(ctx, Q.to(gpu_device), T))
    bad = [8, 9, 10]
    assert np.all(np.isnan(S[:, bad])) and np.all(np.isfinite(np.delete(S, bad, axis=1)))
    Q[0, 5] = float("inf")
    S = f64(als.als_scores(ctx, Q.to(gpu_device), T))
    code = f64(als.als_dequantize(ctx, T))[:, 5]
    ok = np.delete(np.arange(300), bad)
    with np.errstate(all="ignore"):
        assert np.array_equal(S[0, ok], np.where(code[ok] == 0, np.nan, np.inf * code[ok]), equal_nan=True)
    assert np.all(np.isfinite(S[1:, ok]))  # the other queries do not see it


@pytest.mark.parametrize("nq", [1, 2, 4, 40])
@pytest.mark.parametrize("dq", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("big,small", [(127, -20), (-100, 100), (60, -60)])
def test_scores_in_range_of_factors_that_are_not(ctx, gpu_device, nq, dq, big, small):
    say(f"als_scores: queries times 2^{big}, tables times 2^{small}, nq={nq} {dq}")
    for d, group in ((16, 16), (64, 32), (128, 128)):
        T = als.als_quantize(ctx, (init_table(300, d, seed=4, stream=1).clamp(-3, 3) * 2.0 ** small).to(gpu_device), group)
        Q = (init_table(nq, d, seed=6, stream=2).clamp(-1, 1) * 2.0 ** big).to(dq)
        assert torch.all(torch.isfinite(Q))
        S = f64(als.als_scores(ctx, Q.to(gpu_device), T))
        V, Qh = f64(als.als_dequantize(ctx, T)), f64(Q)
        bound = (2 * d + 16) * 2.0 ** -24 * (np.abs(Qh) @ np.abs(V).T)
        assert np.all(np.abs(S - Qh @ V.T) <= bound)


def test_parts_of_a_table_are_tables(ctx, gpu_device):
    say("als_scores: ranges of rows, d=16, 128")
    for d, group in ((16, 16), (128, 32), (64, 16)):
        T = als.als_quantize(ctx, table(1001, d, torch.float32, seed=1, special=False).to(gpu_device), group)
        Q = (init_table(3, d, seed=3, stream=2)).to(gpu_device)
        for nq in (1, 3):
            whole = als.als_scores(ctx, Q[:nq], T)
            part = als.als_scores(ctx, Q[:nq], als.QTable(T.codes[13:900], T.scales[13:900]))
            torch.cuda.synchronize()
            assert torch.equal(whole[:, 13:900], part)


# ------------------------------------------------------------------------------------------------ rules

def lists(rows, cols, mean, gen, values=False, stray=True):
    length = torch.randint(0, 2 * mean + 1, (rows,), generator=gen)
    if rows > 2:
        length[rows // 2] = 0
        length[0] = 3 * mean + 700
    indptr = torch.zeros(rows + 1, dtype=torch.int64)
    indptr[1:] = torch.cumsum(length, 0)
    n = int(indptr[-1])
    ids = (torch.rand(n, generator=gen) ** 4 * cols).to(torch.int32)  # the first items again and again
    if stray and n > 4:
        ids[1], ids[n - 1] = -3, cols
    return indptr, ids, (torch.randn(n, generator=gen) * 8).round() / 8 if values else None


def rules_case(rows, cols, seed, which, exact=False):
    """Keyword arguments of the reference and of binding.Rules (CPU tensors)."""
    gen = torch.Generator().manual_seed(seed)
    kw = {}
    if "h" in which:
        kw["history"] = lists(rows, cols, 9, gen)
        kw.update(dict(repetition=2.0, presence=0.25, frequency=0.125) if exact else dict(repetition=1.3, presence=0.37, frequency=0.11))
    if "p" in which:
        p = torch.rand((rows, 3), generator=gen) + torch.tensor([1.0, 0.0, -0.3])
        kw["penalties"] = torch.tensor([[2.0, 0.5, 0.25], [0.5, 0.0, 0.125]])[torch.arange(rows) % 2] if exact else p
    if "b" in which:
        kw["bias"] = (torch.randn(cols, generator=gen) * 8).round() / 8 if exact else torch.randn(cols, generator=gen)
    if "e" in which:
        kw["entries"] = lists(rows, cols, 5, gen, values=True)
    if "1" in which:
        kw["entries"] = lists(rows, cols, 5, gen)
    if "s" in which or "m" in which:
        words = (cols + 31) // 32
        a = torch.randint(-2 ** 31, 2 ** 31, (rows if "m" in which else 1, words + ("m" in which)), generator=gen).to(torch.int32)
        if "m" in which:
            a[rows // 2] = 0  # nothing is allowed
        kw["allowed"] = a
    return kw


def to_ref(kw):
    out = dict(kw)
    for name in ("history", "entries"):
        if name in out:
            out[name] = tuple(None if t is None else t.numpy() for t in out[name])
    for name in ("penalties", "bias", "allowed"):
        if name in out:
            out[name] = out[name].numpy()
    return out


def to_rules(kw, rows, cols, dev):
    out = dict(kw)
    for name in ("history", "entries"):
        if name in out:
            out[name] = als.Csr(rows, cols, *(None if t is None else t.to(dev) for t in out[name]))
    for name in ("penalties", "bias", "allowed"):
        if name in out:
            out[name] = out[name].to(dev)
    return als.Rules(**out)


SHAPES = [(1, 1), (3, 2), (1, 33), (2, 4095), (5, 4096), (3, 4097), (70, 1031), (4, 20011)]


@pytest.mark.parametrize("which", ["", "h", "hp", "b", "e", "1", "s", "m", "hbes", "hpbem"])
@pytest.mark.parametrize("di,do", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.bfloat16),
                                   (torch.bfloat16, torch.float32)])
def test_adjust_matches_the_definition(ctx, gpu_device, which, di, do):
    for rows, cols in SHAPES:
        say(f"als_adjust {rows} x {cols} rules={which!r} {di} -> {do}")
        gen = torch.Generator().manual_seed(rows + cols)
        X = (torch.randn((rows, cols), generator=gen) * 3).to(di)
        kw = rules_case(rows, cols, rows * cols, which)
        want, mag = ref.adjust(f64(X), **to_ref(kw))
        rules = to_rules(kw, rows, cols, gpu_device)
        bound = 6 * 2.0 ** -24 * mag
        if do == torch.bfloat16:
            bound = bound * 1.01 + np.where(np.isfinite(want), np.abs(want), 0) * 2.0 ** -8
        big = torch.full((rows + 1, cols + 3), 7.0, dtype=do, device=gpu_device)
        got = [big[:rows, 1:cols + 1]]  # rows that start at any element
        als.als_adjust(ctx, strided(X, gpu_device, 1), rules, out=got[0])
        if di == do:
            got.append(als.als_adjust(ctx, X.to(gpu_device), rules))  # in place
        torch.cuda.synchronize()
        for g in got:
            g = f64(g)
            low = np.isneginf(want)
            assert np.array_equal(np.isneginf(g), low)
            with np.errstate(invalid="ignore"):
                assert np.all(np.where(low, 0, np.abs(g - want)) <= bound)
        big[:rows, 1:cols + 1] = 7.0
        assert torch.all(big == 7.0)


def test_adjust_of_special_values(ctx, gpu_device):
    say("als_adjust: infinities, NaN and the lowest value, masked and not")
    X = torch.zeros((2, 96))
    X[:, 0:6] = torch.tensor([float("inf"), float("-inf"), float("nan"), torch.finfo(torch.float32).min, torch.finfo(torch.float32).max, -0.0])
    X[:, 40:46] = X[:, 0:6]
    allowed = torch.full((1, 3), -1, dtype=torch.int32)
    allowed[0, 1] = 0
    bias = torch.zeros(96)
    bias[3] = torch.finfo(torch.float32).min
    got = f64(als.als_adjust(ctx, X.to(gpu_device), als.Rules(allowed=allowed.to(gpu_device), bias=bias.to(gpu_device))))
    assert np.all(np.isneginf(got[:, 32:64]))
    want, _ = ref.adjust(f64(X), bias=bias.numpy(), allowed=allowed.numpy())
    want[:, 3] = -np.inf  # beyond fp32
    assert np.array_equal(got, want, equal_nan=True)


# ------------------------------------------------------------------------------------------------ selection

def check_selected(got, x, k, temperature, n):
    ids, scores, lse = (host(t) for t in got)
    wid, wsc, wl = ref.select(x, k, temperature)
    assert np.array_equal(ids, wid)
    assert np.array_equal(scores.astype(np.float64), wsc)
    for g, w, row in zip(lse.astype(np.float64), wl, x):
        if not np.isfinite(w):
            assert np.array_equal(g, w, equal_nan=True)
        else:
            m = abs(row[row > -np.inf].max()) / temperature
            assert abs(g - w) <= (np.log2(n + 1) + 4) * 2.0 ** -22 + 2.0 ** -22 * (abs(w) + 2 * m)


@pytest.mark.parametrize("which", [None, "h", "hpb", "hbes", "hpbem"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("k,temperature", [(1, 1.0), (20, 0.5), (64, 2.0)])
def test_select_matches_the_definition(ctx, gpu_device, which, dtype, k, temperature):
    for rows, cols in SHAPES + [(1, 300007), (600, 130)]:
        say(f"als_select {rows} x {cols} rules={which!r} {dtype} k={k}")
        gen = torch.Generator().manual_seed(rows + cols)
        # eighths: ties everywhere, and the rules' arithmetic is exact in both widths
        X = ((torch.randn((rows, cols), generator=gen) * 24).round() / 8).to(dtype)
        kw = rules_case(rows, cols, rows * cols, which or "", exact=True)
        want, _ = ref.adjust(f64(X), **to_ref(kw))
        rules = to_rules(kw, rows, cols, gpu_device) if which is not None else None
        got = als.als_select(ctx, strided(X, gpu_device, 3), k, rules, temperature)
        torch.cuda.synchronize()
        check_selected(got, want, k, temperature, cols)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_select_whatever_the_order(ctx, gpu_device, dtype):
    """Equal scores, ascending and descending rows, one value above equal ones, rows with nothing: no order of the scores may
    overflow what is kept or change the answer."""
    n = 50021
    base = torch.arange(n, dtype=torch.float32)
    X = torch.stack([torch.ones(n), base, -base, torch.full((n,), -float("inf")), torch.zeros(n), (base % 97), -(base // 4096)])
    X[4, n - 1] = 1.0
    X[4, ::2] = -0.0
    X[3, 777] = -5.0
    X = X.to(dtype)
    for rows in (slice(0, 7), slice(1, 2), slice(0, 1)):
        for k in (1, 50, 64):
            say(f"als_select orders {dtype} k={k} rows {rows.start}..{rows.stop}")
            got = als.als_select(ctx, X[rows].to(gpu_device).contiguous(), k)
            torch.cuda.synchronize()
            check_selected(got, f64(X[rows]), k, 1.0, n)


def test_select_many_rows_of_ordered_scores(ctx, gpu_device):
    say("als_select 700 x 9000, ascending and equal rows")
    X = torch.arange(9000, dtype=torch.float32)[None, :].repeat(700, 1)
    X[::3] = 2.0
    X[5, 8999] = float("nan")
    got = als.als_select(ctx, X.to(gpu_device), 64)
    torch.cuda.synchronize()
    check_selected(got, f64(X), 64, 1.0, 9000)


def test_select_of_special_values(ctx, gpu_device):
    say("als_select: infinities, NaN, the lowest value")
    low = torch.finfo(torch.float32).min
    X = torch.zeros((6, 5000))
    X[0, 17] = float("inf")
    X[1, 4999] = float("nan")
    X[2] = float("nan")
    X[3] = low
    X[4] = float("-inf")
    X[5] = float("-inf")
    X[5, 9] = float("nan")
    got = als.als_select(ctx, X.to(gpu_device), 3)
    torch.cuda.synchronize()
    check_selected(got, f64(X), 3, 1.0, 5000)
    # a mask takes the NaN and the infinity away
    allowed = torch.full((6, 157), -1, dtype=torch.int32)
    allowed[0, 0] = 0
    allowed[1, 4999 // 32] = 0
    want, _ = ref.adjust(f64(X), allowed=allowed.numpy())
    got = als.als_select(ctx, X.to(gpu_device), 3, als.Rules(allowed=allowed.to(gpu_device)))
    torch.cuda.synchronize()
    check_selected(got, want, 3, 1.0, 5000)


def test_select_without_items_or_rows(ctx, gpu_device):
    say("als_select, als_adjust, als_scores: nothing to do")
    ids, scores, lse = als.als_select(ctx, torch.zeros((3, 0), device=gpu_device), 4)
    torch.cuda.synchronize()
    assert torch.all(ids == -1) and torch.all(scores == -float("inf")) and torch.all(lse == -float("inf"))
    ids, scores, lse = als.als_select(ctx, torch.zeros((0, 8), device=gpu_device), 4)
    assert ids.shape == (0, 4) and lse.shape == (0,)
    assert als.als_adjust(ctx, torch.zeros((0, 8), device=gpu_device), als.Rules()).shape == (0, 8)
    T = als.als_quantize(ctx, torch.zeros((0, 32), device=gpu_device))
    assert als.als_scores(ctx, torch.zeros((2, 32), device=gpu_device), T).shape == (2, 0)
    assert als.als_dequantize(ctx, T).shape == (0, 32)


# ------------------------------------------------------------------------------------------------ together

def test_offsets_beyond_32_bits(ctx, gpu_device):
    say("als_adjust, als_select: rows beyond 2^32 bytes and 2^31 elements")
    cols = 1_100_000_021
    X = torch.zeros((2, cols), dtype=torch.bfloat16, device=gpu_device)
    X[1, cols - 1] = 3.0
    X[1, 5] = 2.0
    X[0, cols - 2] = 1.0
    bias = None
    history = als.Csr(2, cols, torch.tensor([0, 0, 2], device=gpu_device),
                      torch.tensor([cols - 1, 5], dtype=torch.int32, device=gpu_device))
    rules = als.Rules(history=history, repetition=2.0, bias=bias)
    ids, scores, _ = als.als_select(ctx, X, 2, rules)
    als.als_adjust(ctx, X, rules)
    torch.cuda.synchronize()
    assert ids.tolist() == [[cols - 2, 0], [cols - 1, 5]] and scores.tolist() == [[1.0, 0.0], [1.5, 1.0]]
    assert float(X[1, cols - 1]) == 1.5 and float(X[1, 5]) == 1.0 and float(X[0, cols - 2]) == 1.0
    del X
    torch.cuda.empty_cache()


@pytest.mark.parametrize("nq,n", [(40, 130), (1, 70), (2, 300)])
@pytest.mark.parametrize("ds", [torch.float32, torch.bfloat16])
def test_scores_into_rows_far_apart(ctx, gpu_device, nq, n, ds):
    """Rows of scores beyond 2^32 bytes and beyond what a buffer's offsets reach."""
    ld = (1 << 27) + 1 if ds == torch.bfloat16 else (1 << 27) + 2
    say(f"als_scores nq={nq} n={n} ld={ld} {ds}")
    T = als.als_quantize(ctx, table(n, 64, torch.float32, seed=4, special=False).to(gpu_device), 32)
    Q = init_table(nq, 64, seed=3, stream=2).to(gpu_device)
    want = als.als_scores(ctx, Q, T, dtype=ds)
    big = torch.empty(nq * ld, dtype=ds, device=gpu_device)
    S = big.as_strided((nq, n), (ld, 1))
    big.as_strided((nq, n + 3), (ld, 1)).fill_(5.0)
    als.als_scores(ctx, Q, T, out=S)
    torch.cuda.synchronize()
    assert torch.equal(S, want) and torch.all(big.as_strided((nq, 3), (ld, 1), n) == 5.0)
    del S, big
    torch.cuda.empty_cache()


def test_scores_of_many_queries_and_few_items(ctx, gpu_device):
    say("als_scores: 300000 queries x 3 items")
    T = als.als_quantize(ctx, table(3, 16, torch.float32, seed=4, special=False).to(gpu_device), 16)
    Q = init_table(300_000, 16, seed=3, stream=2)
    S = als.als_scores(ctx, Q.to(gpu_device), T)
    torch.cuda.synchronize()
    V = f64(als.als_dequantize(ctx, T))
    want, bound = f64(Q) @ V.T, (2 * 16 + 16) * 2.0 ** -24 * (np.abs(f64(Q)) @ np.abs(V).T) + 1e-37
    assert np.all(np.abs(f64(S) - want) <= bound)


def test_rules_on_many_rows(ctx, gpu_device):
    say("als_select, als_adjust: 70000 rows, more than a grid's second dimension")
    gen = torch.Generator().manual_seed(2)
    X = (torch.randn((70_000, 40), generator=gen) * 8).round() / 8
    got = als.als_select(ctx, X.to(gpu_device), 5)
    Y = als.als_adjust(ctx, X.to(gpu_device), als.Rules(bias=torch.arange(40.0, device=gpu_device)))
    torch.cuda.synchronize()
    check_selected(got, f64(X), 5, 1.0, 40)
    assert np.array_equal(f64(Y), f64(X) + np.arange(40.0))


def serve(ctx, Q, T, rules, k):
    S = als.als_scores(ctx, Q, T)
    als.als_adjust(ctx, S, als.Rules(bias=rules.bias))
    return als.als_select(ctx, S, k, rules)


def test_on_another_stream_and_in_a_graph(ctx, gpu_device):
    say("scores, rules and selection on a side stream and in a replayed graph")
    gen = torch.Generator().manual_seed(4)
    H = table(30011, 64, torch.float32, seed=8, special=False).to(gpu_device)
    Q = torch.randn((24, 64), generator=gen).to(gpu_device)
    rules = to_rules(rules_case(24, 30011, 3, "hbem"), 24, 30011, gpu_device)
    T = als.als_quantize(ctx, H, 32)
    want = serve(ctx, Q, T, rules, 20)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        H2 = H * 1.0  # made on this stream: a call on another one would read it too early
        got = serve(ctx, Q, als.als_quantize(ctx, H2, 32), rules, 20)
    side.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g, w)
    Qs = Q.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = serve(ctx, Qs, T, rules, 20)
    for step in range(4):
        Qs.copy_(Q * (step + 1) if step else Q)
        graph.replay()
        torch.cuda.synchronize()
        again = [t.clone() for t in out]
        want = serve(ctx, Qs, T, rules, 20)
        torch.cuda.synchronize()
        for g, w in zip(again, want):
            assert torch.equal(g, w)


def test_same_bits_every_time(ctx, gpu_device):
    say("als_select, als_scores: the same bits on every call")
    gen = torch.Generator().manual_seed(6)
    X = torch.randn((3, 400_009), generator=gen).to(gpu_device)
    rules = to_rules(rules_case(3, 400_009, 3, "hbem"), 3, 400_009, gpu_device)
    first = als.als_select(ctx, X, 64, rules, 0.7)
    for _ in range(5):
        for a, b in zip(first, als.als_select(ctx, X, 64, rules, 0.7)):
            assert torch.equal(a, b)


def test_a_recorded_request_is_answered_as_a_live_one(ctx, gpu_device):
    say("als_scores, als_adjust, als_select: replayed from a graph")
    gen = torch.Generator().manual_seed(8)
    n, nq = 50_001, 6
    T = als.als_quantize(ctx, torch.randn((n, 64), generator=gen).to(gpu_device))
    Q = torch.randn((nq, 64), generator=gen).to(gpu_device)
    rules = to_rules(rules_case(nq, n, 5, "hbem"), nq, n, gpu_device)
    S, Y = torch.empty((nq, n), device=gpu_device), torch.empty((nq, n), device=gpu_device)

    def request():
        als.als_scores(ctx, Q, T, out=S)
        als.als_adjust(ctx, S, rules, out=Y)
        return als.als_select(ctx, S, 20, rules, 0.9) + als.als_select(ctx, Y, 20)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        request()  # the workspace has its size
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        recorded = request()
    for _ in range(4):
        Q.copy_(torch.randn((nq, 64), generator=gen))
        live = [t.clone() for t in request()] + [Y.clone()]
        S.zero_()
        Y.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(list(recorded) + [Y], live):
            assert torch.equal(a, b)
        assert torch.equal(recorded[0], recorded[3]) and torch.equal(recorded[1], recorded[4])  # the same rules, before or within


def test_the_example_answers_from_4_bits(gpu_device):
    say("examples/serve_4bit.py")
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_4bit.py")
    spec = importlib.util.spec_from_file_location("serve_4bit", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    r = module.main(nodes=12000, epochs=2)
    say(f"  Recall@20 {r['recall'][0]:.4f} from fp32, {r['recall'][1]:.4f} from 4 bits")
    assert r["bytes"][1] * 7 < r["bytes"][0]  # 4.5 bits an entry with groups of 32
    # steps of a seventh of a group's largest entry: an error of about a tenth of an entry, which averages out over a row's 64
    assert r["recall"][1] > 0.8 * r["recall"][0] > 0.04
    ids, prob = r["ids"], r["probability"]
    ptr, idx = r["given"]
    for q in range(0, ids.shape[0], 7):
        assert not set(ids[q].tolist()) & set(idx[ptr[q]:ptr[q + 1]].tolist())
    assert torch.all(prob >= 0) and torch.all(prob.sum(1) <= 1 + 1e-5) and torch.all(prob[:, :-1] >= prob[:, 1:] - 1e-12)


def test_refusals(ctx, gpu_device):
    say("what the operators refuse")
    dev = gpu_device

    def refused(status, f, *args, **kw):
        with pytest.raises(als.AlsError) as e:
            f(ctx, *args, **kw)
        assert e.value.status == status

    H = torch.randn((64, 32), device=dev)
    T = als.als_quantize(ctx, H)
    Q = torch.randn((2, 32), device=dev)
    S = torch.zeros((2, 64), device=dev)
    refused(als.ALS_EDTYPE, als.als_quantize, torch.zeros((4, 48), device=dev), 16)
    refused(als.ALS_ESHAPE, als.als_dequantize, T, out=torch.zeros((63, 32), device=dev))
    refused(als.ALS_ESHAPE, als.als_dequantize, T, out=torch.zeros((64, 64), device=dev))
    refused(als.ALS_ESHAPE, als.als_scores, torch.zeros((2, 64), device=dev), T)
    refused(als.ALS_ESHAPE, als.als_scores, Q, T, out=torch.zeros((2, 63), device=dev))
    refused(als.ALS_ESHAPE, als.als_scores, Q, als.QTable(T.codes.view(-1)[1:].view(-1)[: 63 * 16].view(63, 16), T.scales[:63]))
    both = torch.zeros((4, 64), device=dev)
    refused(als.ALS_EALIAS, als.als_adjust, both[:2], als.Rules(), out=both[1:3])
    refused(als.ALS_EALIAS, als.als_adjust, S, als.Rules(bias=both[0]), out=both[:2])
    refused(als.ALS_ESHAPE, als.als_adjust, S, als.Rules(), out=torch.zeros((2, 65), device=dev))
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        refused(als.ALS_EINVAL, als.als_adjust, S, als.Rules(repetition=bad))
        refused(als.ALS_EINVAL, als.als_select, S, 3, temperature=bad)
    refused(als.ALS_EINVAL, als.als_adjust, S, als.Rules(presence=float("nan")))
    refused(als.ALS_EINVAL, als.als_select, S, 0)
    refused(als.ALS_EINVAL, als.als_select, S, 65)
    short = als.Csr(1, 64, torch.zeros(2, dtype=torch.int64, device=dev), torch.zeros(0, dtype=torch.int32, device=dev))
    refused(als.ALS_ESHAPE, als.als_adjust, S, als.Rules(history=short))
    refused(als.ALS_ESHAPE, als.als_select, S, 3, als.Rules(entries=short))
    refused(als.ALS_ESHAPE, als.als_select, S[:, :1].expand(2, 64)[:, :64].as_strided((2, 64), (1, 1)), 3)
    torch.cuda.synchronize()
