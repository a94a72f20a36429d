"""Host checks of the operators over ordered histories: what the binding refuses before anything reaches the GPU, a null
context, and the references on numbers done by hand and against each other."""
import ctypes
import os

import numpy as np
import pytest
import torch

import history_ref as ref
from paper_2112_02194_amd import binding as als


class HostContext:
    """Stands for a context where no call may get as far as the library."""
    device = torch.device("cuda", 0)


def test_lists_without_ids():
    y = als.Csr(2, 5, torch.tensor([0, 2, 5]), None)
    c = y.c()
    assert y.nnz == 5 and (c.rows, c.cols, c.nnz, c.indices, c.values) == (2, 5, 5, None, None)


def test_what_the_binding_refuses():
    ctx, z = HostContext(), torch.zeros
    with pytest.raises(ValueError):
        als.als_beam(ctx, z((6, 3), dtype=torch.int32), z((6, 3)), z(6), z(6), 4)
    with pytest.raises(ValueError):
        als.als_beam(ctx, z((6, 3), dtype=torch.int64), z((6, 3)), z(6), z(6), 3)
    with pytest.raises(ValueError):
        als.als_beam(ctx, z((6, 3), dtype=torch.int32), z((6, 2)), z(6), z(6), 3)
    for bad in (dict(lse=z(5)), dict(totals=z(6, dtype=torch.float64)), dict(last=z(6)), dict(lengths=z((6, 1), dtype=torch.int32)),
                dict(factors=z((2, 2))), dict(factors=z(0))):
        with pytest.raises(ValueError):
            als.als_beam(ctx, z((6, 3), dtype=torch.int32), z((6, 3)), **{"lse": z(6), "totals": z(6), **bad}, beams=3)
    parents = z(6, dtype=torch.int32)
    for bad in ([z((5, 2))], [z((6, 4))[:, ::2]], [z((6, 4, 4)).transpose(1, 2)]):
        with pytest.raises(ValueError):
            als.als_reorder(ctx, parents, 3, bad)
    with pytest.raises(ValueError):
        als.als_reorder(ctx, parents, 4, [])
    with pytest.raises(TypeError):
        als.als_reorder(ctx, parents, 3, [z((6, 4), dtype=torch.uint8)])
    with pytest.raises(ValueError):
        als.als_reorder(ctx, parents, 3, [z((6, 4))], out=[z((6, 4), dtype=torch.bfloat16)])
    with pytest.raises(TypeError):
        als.als_clip(ctx, [z(3, dtype=torch.float64)], 1.0)
    with pytest.raises(ValueError):
        als.als_clip(ctx, [z(3)], 1.0, out=[z(4)])
    with pytest.raises(ValueError):
        als.als_clip(ctx, [z((4, 4)).t()], 1.0)
    with pytest.raises(ValueError):  # not on the context's GPU
        als.als_clip(ctx, [z(3)], 1.0)
    with pytest.raises(ValueError):
        als.als_sum_rows(ctx, als.Csr(1, 2, torch.tensor([0, 0]), z(0, dtype=torch.int32)), z((2, 16)))
    with pytest.raises(ValueError):
        als.als_recur_step(ctx, parents, z((2, 16)), z((2, 16)), z((6, 16)), out=z((5, 16)))


def test_a_state_of_any_shape_is_a_row_a_beam():
    words = lambda t, rows: als._states(-1, [t], rows).tolist()[1:]  # noqa: E731
    assert words(torch.zeros((6, 3, 4, 2), dtype=torch.int64), 6) == [6, 48, 48, als.ALS_F32]
    assert words(torch.zeros((6, 10), dtype=torch.float16)[:, :7], 6) == [6, 7, 10, als.ALS_BF16]
    assert words(torch.zeros((1, 5), dtype=torch.int32), 1) == [1, 5, 5, als.ALS_F32]
    assert words(torch.zeros(4), 4) == [4, 1, 1, als.ALS_F32]
    assert words(torch.zeros((3, 0)), 3) == [3, 0, 0, als.ALS_F32]


def test_tensors_as_rows_of_values():
    assert als._flat_values(-1, [torch.zeros((2, 3)), torch.zeros(0, dtype=torch.bfloat16)]).tolist()[1:5] == [1, 6, 6, als.ALS_F32]
    assert als._flat_values(-1, []).tolist() == []
    assert als._row_values(-1, [torch.zeros((4, 6))[:, :3]]).tolist()[1:] == [4, 3, 6, als.ALS_F32]


def test_null_context():
    if not os.path.exists(als.LIB_PATH):
        pytest.skip("library not built")
    lib = als.load_library()
    assert lib.als_recur(None, None, None, None, None, None, None, None) == als.ALS_EINVAL
    assert lib.als_recur_step(None, None, None, None, None, None, None, None) == als.ALS_EINVAL
    assert lib.als_recur_backward(*[None] * 12) == als.ALS_EINVAL
    assert lib.als_sum_rows(None, None, None, None, None) == als.ALS_EINVAL
    assert lib.als_clip(None, None, None, 0, 1.0, None, None) == als.ALS_EINVAL
    assert lib.als_beam(None, None, None, None, None, None, None) == als.ALS_EINVAL
    assert lib.als_reorder(None, None, 0, 1, None, None, 0, None) == als.ALS_EINVAL
    assert ctypes.sizeof(als.c_als_matrix) == 40  # five words of 64 bits, as als_clip's arrays are filled


def test_references_on_numbers_done_by_hand():
    V, F = np.array([[4.0], [-2.0]]), np.array([[0.0], [np.log(3.0)]])  # s = 1/2, 3/4
    last, states, _, _ = ref.recur([0, 0, 3], [0, 1, 7], V, F, np.array([[5.0], [8.0]]))
    assert np.allclose(last[:, 0], [5.0, 4.0]) and np.allclose(states[:, 0], [6.0, 4.0, 4.0])
    (dV, dF, dH0), _ = ref.recur_backward([0, 0, 3], [0, 1, 7], V, F, states, d_last=np.array([[9.0], [1.0]]), H0=np.array([[5.0], [8.0]]))
    assert np.allclose(dV[:, 0], [0.375, 0.25, 0.0]) and np.allclose(dH0[:, 0], [9.0, 0.375])
    assert np.allclose(dF[:, 0], [0.75 * 4.0 * 0.25, 8.0 * 0.1875, 0.0])
    X, _ = ref.sum_rows([0, 2, 2, 3], [0, 1, -1], [2.0, 1.0, 5.0], V)
    assert X[:, 0].tolist() == [6.0, 0.0, 0.0]
    f = np.float32
    got = ref.beam(np.array([[3, 4], [5, -1]]), np.array([[2, 1], [4, 9]], dtype=f), np.array([1, 2], dtype=f), np.array([0, -1], dtype=f), 2)
    assert got[0].tolist() == [0, 1] and got[1].tolist() == [3, 5] and got[2].tolist() == [1.0, 1.0] and got[3].tolist() == [1, 1]
    got = ref.beam(np.array([[3, 4], [5, 6]]), np.array([[2, 1], [4, 3]], dtype=f), None, np.array([0, -9], dtype=f), 2, last=np.array([7, 0]), end=7)
    assert got[0].tolist() == [0, 1] and got[1].tolist() == [7, 5] and got[2].tolist() == [0.0, -5.0] and got[3].tolist() == [0, 1]


def test_the_reference_gradients_are_differences_of_the_reference():
    rng = np.random.default_rng(3)
    V, F, H0 = rng.normal(size=(5, 2)), rng.normal(size=(5, 2)), rng.normal(size=(4, 2))
    ptr, ids = np.array([0, 3, 3, 4, 9]), np.array([0, 4, 4, 2, 1, 0, 9, 3, 4])
    ws, wl = rng.normal(size=(9, 2)), rng.normal(size=(4, 2))

    def loss(V, F, H0):
        last, states, _, _ = ref.recur(ptr, ids, V, F, H0)
        return (ws * states).sum() + (wl * last).sum()

    (dV, dF, dH0), _ = ref.recur_backward(ptr, ids, V, F, ref.recur(ptr, ids, V, F, H0)[1], ws, wl, H0)
    ok = ids < 5
    gV, gF = np.zeros_like(V), np.zeros_like(F)
    np.add.at(gV, ids[ok], dV[ok])
    np.add.at(gF, ids[ok], dF[ok])
    for name, grad in (("V", gV), ("F", gF), ("H0", dH0)):
        for at in np.ndindex(grad.shape):
            args = {"V": V, "F": F, "H0": H0}
            step = np.zeros_like(grad)
            step[at] = 1e-5
            up, down = (loss(**{**args, name: args[name] + s * step}) for s in (1, -1))
            assert abs((up - down) / 2e-5 - grad[at]) < 1e-8
