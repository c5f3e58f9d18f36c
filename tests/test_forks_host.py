"""Forks of requests as an engine makes them, on the host: none at all, and numbers that no row has."""
import numpy as np
import pytest

from paper_2609_31395_amd import actkv


@pytest.mark.parametrize("lens", [[], np.zeros((0, 4)), np.zeros((0, 4), np.int32), np.zeros(0)])
@pytest.mark.parametrize("share", [True, False])
def test_no_forks_of_lengths(lens, share):
    f = actkv.Forks.of_lengths([], [], lens, share)
    assert f.host.shape == (0, 4) and f.num_fresh == 0


def test_lengths_without_a_fork_are_refused():
    with pytest.raises(ValueError):
        actkv.Forks.of_lengths([], [], [[3, 4]])
    with pytest.raises(ValueError):
        actkv.Forks.of_lengths([0], [1], [])


@pytest.mark.parametrize("bad", [np.array([1 << 32]), np.array([(1 << 32) + 1]), [1 << 31], [-(1 << 31) - 1], [1.5], [float("nan")],
                                 [float("inf")], np.array([3e9])])
@pytest.mark.parametrize("column", ["parents", "children", "shared", "pages"])
def test_numbers_that_no_row_has_are_refused(column, bad):
    cols = dict(parents=[0], children=[1], shared=[0], pages=[0])
    cols[column] = bad
    with pytest.raises(ValueError, match=column):
        actkv.Forks(**cols)


@pytest.mark.parametrize("good", [[2], [2.0], np.array([2], np.int64), np.array([2], np.uint8), np.array([[2]])])
def test_whole_numbers_of_any_type(good):
    f = actkv.Forks(good, [1], [0], good)
    assert f.host.tolist() == [[2, 1, 0, 2]] and f.host.dtype == np.int32
    f = actkv.Forks.of_lengths([0], [1], np.array([[40, 64]], np.int64))
    assert f.host.tolist() == [[0, 1, 2, 4]]
