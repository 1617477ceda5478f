"""The distillation oracle on rows whose largest logit dwarfs the logarithm of the sum."""

import numpy as np

from oracle import sequence as seq


def test_uniform_row_at_the_lowest_value():
    # every logit the lowest float32: each place has probability 1 / V
    V, q = 50, np.array([0.5, 0.25, 0.25])
    z = np.full((1, V), np.finfo(np.float32).min, dtype=np.float64)
    loss, gz = seq.distill(z, np.array([[3, 8, 20]]), np.log(q)[None], labels=np.array([8]), alpha=0.25)
    assert np.isclose(loss[0], 0.75 * np.log(V) + 0.25 * (q * (np.log(q) + np.log(V))).sum(), rtol=1e-14)
    want = np.full(V, 1 / V)
    want[[3, 8, 20]] -= 0.25 * q
    want[8] -= 0.75
    assert np.allclose(gz[0], want, rtol=1e-14, atol=1e-16)


def test_row_of_tiny_and_lowest_values():
    z = np.array([[np.finfo(np.float32).min, 0.5, -0.25, -np.inf]])
    loss, gz = seq.distill(z, np.array([[1, 2]]), np.array([[1.0, 0.0]]), temperature=2.0)
    p, q = np.exp([0.25, -0.125]), np.exp([0.5, 0.0])
    p, q = p / p.sum(), q / q.sum()
    assert np.isclose(loss[0], 4 * (q * (np.log(q) - np.log(p))).sum(), rtol=1e-13)
    assert np.allclose(gz[0], [0, *(2 * (p - q)), 0], rtol=1e-13, atol=1e-16)
