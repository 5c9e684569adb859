"""The oracle's sampler and acceptance on rows without a value above -inf: the
lowest index of -inf, 0 when every value is NaN."""
import numpy as np

from oracle import filter as of

N, M = np.nan, -np.inf


def test_sampler_and_acceptance():
    for row, want in (([N, N, N], 0), ([M, M], 0), ([N, M, M], 1), ([N, N, N, M], 3), ([N], 0)):
        assert of.sample(row, 0.5) == (want, 0.0)
        z = np.array([row, row])
        p = np.zeros(z.shape)
        assert of.accept(p, p[:1], [0], [0.5, 0.5], z) == (0, want)


def test_second_row_without_a_number():
    z = np.array([[0.0, 1.0, 2.0], [N, M, N]])
    p = np.array([of.probs(of.kept_weights(r)) for r in z])
    assert of.accept(p, p[:1], [2], [0.9, 0.3], z) == (1, 1)
