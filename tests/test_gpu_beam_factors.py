"""als_beam where factors are negative, zero, infinite or NaN: what is no candidate stays none.  Equal to the definition to the bit."""
import numpy as np
import pytest
import torch

import beam_ref
from gpu_util import say
from paper_2112_02194_amd import binding as als

pytestmark = pytest.mark.gpu

FACTORS = {"negative": [-1.0, -0.5, -2.0, -0.25], "mixed": [1.0, -1.0, 0.0, 0.5], "zero": [0.0], "odd": [-1.0, float("nan"), float("inf"), -float("inf")]}


@pytest.fixture(scope="module")
def ctx(gpu_device):
    c = als.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("factors", list(FACTORS))
@pytest.mark.parametrize("kind", ["plain", "first step", "ended", "few", "dead beams"])
@pytest.mark.parametrize("groups,beams,k", [(1, 1, 1), (3, 4, 5), (2, 64, 3), (2, 64, 64), (70, 50, 64)])
def test_candidates_by_the_definition(ctx, gpu_device, groups, beams, k, kind, factors):
    say(f"als_beam {groups} x {beams} x {k}, {kind}, {factors} factors")
    gen = np.random.default_rng(11)
    rows, f = groups * beams, np.float32
    ids = gen.integers(0, 1000, (rows, k)).astype(np.int32)
    scores, lse, totals = (gen.normal(size=s).astype(f) for s in ((rows, k), rows, rows))
    last, lengths = np.full(rows, 7, dtype=np.int32), gen.integers(0, 6, rows).astype(np.int32)
    if kind == "few":
        ids[gen.random(ids.shape) < 0.8] = -1
        scores[gen.random(scores.shape) < 0.1] = np.nan
    if kind == "dead beams":
        totals[gen.random(rows) < 0.6] = -np.inf
        totals[gen.random(rows) < 0.1] = np.nan
    if kind == "ended":
        last[gen.random(rows) < 0.5] = 0
        totals[gen.random(rows) < 0.2] = -np.inf
    args = dict(last=last, end=0, lengths=lengths, factors=np.array(FACTORS[factors], dtype=f))
    before = None if kind == "first step" else totals
    want = beam_ref.beam(ids, scores, lse, before, beams, temperature=0.7, **args)
    dev = {n: torch.from_numpy(v).to(gpu_device) if isinstance(v, np.ndarray) else v for n, v in args.items()}
    put = lambda a: None if a is None else torch.from_numpy(a).to(gpu_device)  # noqa: E731
    got = als.als_beam(ctx, put(ids), put(scores), put(lse), put(before), beams, temperature=0.7, **dev)
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert np.array_equal(g.cpu().numpy(), w)
