"""A row of more than 2^31 entries, whose pieces fill the workspace: every piece counts once, in its place."""
import numpy as np
import pytest
import torch

from gpu_util import f64, say
from paper_2112_02194_amd import binding as als
from test_gpu_history import F32

pytestmark = pytest.mark.gpu
N = (1 << 31) + 70_001
BLOCK = 1 << 15  # below half a chunk: 32768 chunks hold N entries


@pytest.fixture(scope="module")
def ctx(gpu_device):
    c = als.Context(0)
    yield c
    c.close()


def rows_of(ids, cols):
    """A row of one entry, the long one, a short one."""
    return als.Csr(3, cols, torch.tensor([0, 1, N - 300, N], device=ids.device), ids)


def test_every_stretch_is_summed_once(ctx, gpu_device):
    """One entry in every 32768 has a vector, the number of its stretch in bits and a one; the others are zeros.  All sums are whole
    numbers below 2^24, exact in fp32 in any order: a stretch that is lost or taken twice shows, and which."""
    say(f"als_sum_rows: {N} entries, a marked one in every {BLOCK}")
    blocks = (N - 300) // BLOCK
    number = torch.arange(blocks)
    E = torch.zeros((blocks + 1, 32))
    E[1:, :17] = (number[:, None] >> torch.arange(17) & 1).float()
    E[1:, 17] = 1.0
    ids = torch.zeros(N, dtype=torch.int32, device=gpu_device)
    place = torch.randint(1, BLOCK, (blocks,), generator=torch.Generator().manual_seed(1))
    ids[(number * BLOCK + place).to(gpu_device)] = (number + 1).to(torch.int32).to(gpu_device)
    X = als.als_sum_rows(ctx, rows_of(ids, blocks + 1), E.to(gpu_device)).cpu()
    assert blocks < 2 ** 17 and torch.all(E.double().sum(0) < 2 ** 24)
    assert torch.equal(X[1].double(), E.double().sum(0))
    assert torch.all(X[0] == 0) and torch.all(X[2] == 0)
    del ids
    torch.cuda.empty_cache()


def test_every_piece_is_walked_in_its_place(ctx, gpu_device):
    """Entries without an item but for 128 marked ones, whose gates keep 63/64; in column c the marked entries 16 k + c have the value 1, the
    others 0.  So h_c = sum of (1/64) (63/64)^(marked entries behind) over its own.  Of a marked entry that is lost, doubled or moved past
    another, column c shows at least (1/64) (63/64)^127 / 64 = 3e-5, or 3e-4 of h_c, which is below 0.09.

    fp32: each marked entry is some roundings of h_c and of its map where it stands, and each of the up to 256 pieces after each other and 128 stretches
    of pieces of the join, where nothing is rounded for a piece without a mark (its map is exactly the identity): 128 * (4 + 13) u, 13 u the
    gate's bound at |F| = 4.1, is 1.3e-4 of h_c."""
    say(f"als_recur: {N} entries, 128 with an item")
    d, marks = 16, 128
    gen = torch.Generator().manual_seed(2)
    at = torch.sort(torch.cat([torch.randint(1, N - 300, (marks - 4,), generator=gen), torch.tensor([1, (1 << 31) - 1, 1 << 31, N - 301])])).values
    assert at.unique().numel() == marks
    V, F = torch.eye(16), torch.full((16, d), float(np.log(63.0)))
    ids = torch.full((N,), -1, dtype=torch.int32, device=gpu_device)
    ids[at.to(gpu_device)] = (torch.arange(marks) % 16).to(torch.int32).to(gpu_device)
    last, _ = als.als_recur(ctx, rows_of(ids, 16), V.to(gpu_device), F.to(gpu_device))
    s = 1 / (1 + np.exp(-f64(F)[0, 0]))
    weight = (1 - s) * s ** np.arange(marks - 1, -1, -1.0)
    want = np.array([weight[c::16].sum() for c in range(16)])
    off = np.abs(f64(last)[1] - want)
    print(off / want)
    assert np.all(off <= 128 * 17 * 2.0 ** -24 * want)
    assert torch.all(last[[0, 2]] == 0)
    del ids
    torch.cuda.empty_cache()
