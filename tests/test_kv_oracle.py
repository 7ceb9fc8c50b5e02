"""Page selection's definition (oracle/kv_oracle.py) where scores are no numbers (CPU only)."""
import numpy as np
import pytest

from oracle import kv_oracle as O


@pytest.mark.parametrize("flip", [False, True])
def test_a_head_whose_sum_is_no_number_is_passed_over(flip):
    # head 0 meets 0 * inf everywhere on pages 1 and 2, head 1 has 5 and 6 there: whichever comes first
    q = np.array([[np.inf, 1.0], [1.0, 1.0]])
    lo, hi = np.zeros((5, 2)), np.array([[9.0, 9], [0, 5], [0, 6], [1, 3], [9, 9]])
    lo[:, 0] = hi[:, 0] = 0.0
    hi[0, 0] = hi[4, 0] = 1.0
    assert O.choose(q[::-1] if flip else q, lo, hi, 5, 3, 1, 1) == [0, 2, 4]
    lo[2, 0], hi[2, 0] = np.nan, np.nan                                # no head has a number: last
    assert O.choose(q[::-1] if flip else q, lo, hi, 5, 3, 1, 1) == [0, 1, 4]


def test_a_page_with_a_dimension_without_numbers_comes_last():
    rng = np.random.default_rng(0)
    for value in (2.0, -2.0, 0.0):
        q = rng.standard_normal((3, 4))
        q[:, 1] = value
        lo = -np.abs(rng.standard_normal((9, 4)))
        hi = -lo
        lo[3, 1], hi[3, 1] = np.inf, -np.inf
        for n in range(3, 9):  # eight pages at most: page 3 is the one left out
            assert 3 not in O.choose(q, lo, hi, 9, n, 1, 1)
        hi[3, 2] = np.inf      # nor does a key that is +inf elsewhere bring it back
        assert 3 not in O.choose(q, lo, hi, 9, 8, 1, 1)


def test_infinite_summaries_that_a_query_does_not_meet():
    # a zero of the query takes k_min: +inf in k_max is not met, -inf in k_min is
    q = np.array([[0.0, 1.0]])
    lo, hi = np.array([[0.0, 0], [-1, 1], [-1, 2], [-np.inf, 9], [0, 0]]), np.array([[0.0, 0], [np.inf, 7], [1, 6], [1, 9], [0, 0]])
    assert O.choose(q, lo, hi, 5, 3, 1, 1) == [0, 1, 4]
