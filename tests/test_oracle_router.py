"""The router's oracle: closed forms, ties and masks, and its gradient against differences (CPU only)."""

import numpy as np
import pytest

from oracle import router

MODES = [(s, n) for s in ("softmax", "sigmoid") for n in (False, True)]


def test_choice_ties_masks_and_nan():
    z = np.array([[1.0, 3.0, 3.0, -np.inf, 2.0], [-np.inf] * 5, [np.nan, 0.0, -np.inf, 0.0, -1.0]])
    assert router.choose(z, None, 4, "softmax").tolist() == [[1, 2, 4, 0], [-1] * 4, [1, 3, 4, -1]]
    # a bias turns the choice, a masked expert stays out, equal sums go to the lower index
    assert router.choose(z[:1], np.array([0.0, 0.0, 0.0, 9.0, 5.0]), 2, "sigmoid").tolist() == [[4, 1]]


@pytest.mark.parametrize("score,normalize", MODES)
def test_weights_sum(score, normalize):
    z = np.random.default_rng(0).normal(size=(7, 9))
    idx = router.choose(z, None, 9, score)
    w = router.weights(z, idx, score, normalize, 2.5)
    if score == "softmax" or normalize:
        assert np.allclose(w.sum(axis=1), 2.5, rtol=1e-14)
    else:
        assert np.allclose(np.sort(w, axis=1), np.sort(2.5 / (1 + np.exp(-z)), axis=1), rtol=1e-14)


def test_normalized_sigmoid_of_tiny_scores():
    w = router.weights(np.array([[-800.0, -801.0, -900.0]]), np.array([[0, 1]]), "sigmoid", True, 1.0)
    assert np.allclose(w, [[1 / (1 + np.exp(-1.0)), 1 / (1 + np.exp(1.0))]], rtol=1e-12)


@pytest.mark.parametrize("score,normalize", MODES)
def test_gradient_against_differences(score, normalize):
    rng = np.random.default_rng(1)
    z = rng.normal(size=(5, 6))
    idx = router.choose(z, None, 3, score)
    idx[2, 2] = -1
    idx[3] = [1, 1, -1]  # the same expert twice
    dp = rng.normal(size=(5, 3))
    got = router.weights_bwd(z, idx, dp, score, normalize, 2.5)
    h = 1e-5
    for i in range(6):
        d = np.zeros_like(z)
        d[:, i] = h
        f = lambda v: (router.weights(v, idx, score, normalize, 2.5) * dp).sum(axis=1)  # noqa: E731
        # central differences: h^2 / 6 times a third derivative of at most about 10, and rounding 1e-16 / h
        assert np.allclose((f(z + d) - f(z - d)) / (2 * h), got[:, i], atol=1e-8)
