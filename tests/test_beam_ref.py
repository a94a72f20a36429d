"""The definition of als_beam's candidates on numbers done by hand."""
import numpy as np

import beam_ref

f = np.float32


def test_an_id_that_is_none_stays_none_where_a_factor_is_negative():
    """Row 0: one item with total 1 - 2 = -1; row 1 has no items.  A factor of -1 orders by 1; the places without an item
    are no candidates, whatever -inf times the factor is."""
    got = beam_ref.beam(np.array([[4, -1], [-1, -1]]), np.array([[-2, 0], [5, 4]], dtype=f), None, np.array([1, 3], dtype=f), 2,
                        factors=np.array([1, -1], dtype=f))
    assert [g.tolist() for g in got] == [[0, -1], [4, -1], [-1.0, -np.inf], [1, 0]]


def test_an_ended_beam_has_one_candidate_where_a_factor_is_negative():
    """Both beams have ended, with lengths 1 and 0: keys 2 * -1 and -3 * 1."""
    got = beam_ref.beam(np.array([[4, 5], [6, 7]]), np.zeros((2, 2), dtype=f), None, np.array([2, -3], dtype=f), 2, last=np.array([9, 9]), end=9,
                        lengths=np.array([1, 0]), factors=np.array([1, -1], dtype=f))
    assert [g.tolist() for g in got] == [[0, 1], [9, 9], [2.0, -3.0], [1, 0]]


def test_the_first_step_has_one_beam_where_a_factor_is_negative():
    got = beam_ref.beam(np.array([[4], [6]]), np.array([[-5], [-1]], dtype=f), None, None, 2, factors=np.array([1, -1], dtype=f))
    assert [g.tolist() for g in got] == [[0, -1], [4, -1], [-5.0, -np.inf], [1, 0]]
