"""The drafting oracle on rows without a distribution. CPU only."""

import numpy as np
import pytest

from oracle import drafting as dra

N, I = np.nan, np.inf


@pytest.mark.parametrize("row,greedy,drawn", [
    ([-I, -I, -I], 0, -1), ([N, N, -I], 2, -1), ([N, N, N], -1, -1), ([0.0, I, I], 1, -1),
    ([N, -1.0, -2.0], 1, -1), ([1.0, 1.0, -I], 0, 0)])
def test_next_token(row, greedy, drawn):
    """0 is the random number; infinities are numbers to a temperature of 0 alone."""
    x = np.array([row], np.float32)
    for temperature, want in ((0.0, greedy), (1.0, drawn)):
        counts, following, paths, _ = dra.verify(x, [0], [0, 1], 1, np.zeros(1, np.float32),
                                                 temperature=temperature)
        assert (counts[0], following[0], paths[0].tolist()) == (0, want, [0, -1])
