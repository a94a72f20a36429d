"""Host checks of the operators that answer from trained tables: what the binding refuses before anything reaches the GPU,
a null context, and the references against each other on small numbers."""
import os

import numpy as np
import pytest
import torch

import serving_ref as ref
from paper_2112_02194_amd import binding as als


def test_qtable_shapes_and_refusals():
    T = als.QTable(torch.zeros((5, 32), dtype=torch.uint8), torch.zeros((5, 2), dtype=torch.bfloat16))
    assert T.shape == (5, 64) and T.group == 32
    c = T.c()
    assert (c.rows, c.d, c.group) == (5, 64, 32)
    with pytest.raises(TypeError):
        als.QTable(T.codes.int(), T.scales).c()
    with pytest.raises(TypeError):
        als.QTable(T.codes, T.scales.float()).c()
    with pytest.raises(ValueError):
        als.QTable(T.codes[:, :16], T.scales).c()
    with pytest.raises(ValueError):
        als.QTable(T.codes, T.scales[:4]).c()


def test_rules_shapes_and_refusals():
    a = torch.zeros((3, 4), dtype=torch.int32)
    assert als.Rules(allowed=a).c(3, 97).allowed_ld == 4
    assert als.Rules(allowed=a[:1]).c(3, 97).allowed_ld == 0
    assert als.Rules(allowed=a[:1].expand(3, 4)).c(3, 97).allowed_ld == 0
    for bad in (dict(allowed=a[:2]), dict(allowed=a[:, :3]), dict(allowed=a.long()), dict(bias=torch.zeros(96)),
                dict(bias=torch.zeros(97, dtype=torch.float64)), dict(penalties=torch.zeros((3, 2)))):
        with pytest.raises(ValueError):
            als.Rules(**bad).c(3, 97)


def test_scores_matrix_refusals():
    assert als._matrix(torch.zeros((1, 7))).ld == 7
    assert als._matrix(torch.zeros((4, 9))[:, 1:8]).ld == 9
    with pytest.raises(ValueError):
        als._matrix(torch.zeros((4, 9)).T)
    with pytest.raises(TypeError):
        als._matrix(torch.zeros((4, 9), dtype=torch.float16))
    with pytest.raises(ValueError):
        als.als_quantize(None, torch.zeros((4, 16)), 32)


class NoCalls:
    """Context of GPU 0 whose library must not be reached."""
    device, handle = torch.device("cuda", 0), None


def test_tensors_elsewhere_are_refused():
    T = als.QTable(torch.zeros((5, 16), dtype=torch.uint8), torch.zeros((5, 1), dtype=torch.bfloat16))
    X, S = torch.zeros((5, 32)), torch.zeros((2, 5))
    lists = als.Csr(2, 5, torch.zeros(3, dtype=torch.int64), torch.zeros(0, dtype=torch.int32))
    for call in (lambda c: als.als_quantize(c, X), lambda c: als.als_dequantize(c, T), lambda c: als.als_scores(c, X, T),
                 lambda c: als.als_adjust(c, S, als.Rules()), lambda c: als.als_select(c, S, 1),
                 lambda c: als.als_select(c, S, 1, als.Rules(history=lists, bias=torch.zeros(5)))):
        with pytest.raises(ValueError, match="GPU"):
            call(NoCalls())
    assert len(als.Rules(history=lists, entries=lists).tensors()) == 9


def test_null_context_is_refused():
    if not os.path.exists(als.LIB_PATH):
        pytest.skip("library not built")
    lib = als.load_library()
    assert lib.als_quantize(None, None, None, None) == als.ALS_EINVAL
    assert lib.als_dequantize(None, None, None, None) == als.ALS_EINVAL
    assert lib.als_scores(None, None, None, None, None) == als.ALS_EINVAL
    assert lib.als_adjust(None, None, None, None, None) == als.ALS_EINVAL
    assert lib.als_select(None, None, None, 1.0, 1, None, None, None, None) == als.ALS_EINVAL


def test_references_on_numbers_done_by_hand():
    code, scale = ref.quantize(np.array([[7.0, -3.4, 0.0, 0.5] * 4], dtype=np.float32), 16)
    assert scale.tolist() == [[1.0]] and code[0, :4].tolist() == [7, -3, 0, 0]
    assert ref.pack(code)[0, :2].tolist() == [0xD7, 0x00]
    x, _ = ref.adjust(np.array([[2.0, -2.0, 1.0]]), history=(np.array([0, 3]), np.array([0, 1, 1])), repetition=2.0, presence=0.5,
                      frequency=0.25, allowed=np.array([[3]], dtype=np.int32))
    assert x.tolist() == [[0.25, -5.0, -np.inf]]
    ids, scores, lse = ref.select(np.array([[1.0, 3.0, 3.0, -np.inf]]), 4)
    assert ids.tolist() == [[1, 2, 0, -1]] and scores[0, :3].tolist() == [3.0, 3.0, 1.0]
    assert abs(lse[0] - np.log(2 * np.exp(3.0) + np.exp(1.0))) < 1e-12
