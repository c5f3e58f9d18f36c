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
