"""Pins of the oracle's adapter objective: its gradient against differences of its loss, and against the full softmax regression
whose matrix it factors."""
import numpy as np
import pytest

from oracle import objectives as ob
from rfast_workloads import problems
from rfast_workloads.problems import bf16_bits_to_f32


def _make(rounding, d=20, K=7, rank=3, seed=1):
    data = problems.lora_softmax(3, d, K, rank, 24, seed)
    X = bf16_bits_to_f32(data["Xb"])
    return ob.LoraSoftmax(X, data["labels"], bf16_bits_to_f32(data["W0"]), rank, 0.6, rounding), data["x0"].astype(np.float64), X


def test_gradient_against_differences():
    obj, x0, _ = _make(False)
    obj.lab[1][3] = -1
    rng = np.random.default_rng(0)
    for i in range(3):
        g = obj.grad(i, x0[i], 0)
        for _ in range(4):
            v = rng.standard_normal(obj.p)
            h = 1e-5
            diff = (obj.loss(i, x0[i] + h * v) - obj.loss(i, x0[i] - h * v)) / (2 * h)
            assert abs(diff - g @ v) <= 1e-7 * (1 + abs(diff))


@pytest.mark.parametrize("batch", [None, [3, 3, 0, 17]])
def test_gradient_is_the_full_one_through_the_factors(batch):
    obj, x0, X = _make(False)
    A, B = x0[0][:60].reshape(3, 20), x0[0][60:].reshape(7, 3)
    W = obj.W0 + 0.6 * B @ A                     # K x d
    rows = np.arange(24) if batch is None else np.array(batch)
    logits = X[0][rows].astype(np.float64) @ W.T
    P = np.exp(logits) / np.exp(logits).sum(1, keepdims=True)
    P[np.arange(len(rows)), obj.lab[0][rows]] -= 1
    G = P.T @ X[0][rows] / len(rows)             # of W
    want = np.concatenate([(0.6 * B.T @ G).reshape(-1), (0.6 * G @ A.T).reshape(-1)])
    assert np.allclose(obj.grad(0, x0[0], 0, batch), want, rtol=1e-12, atol=1e-15)


def test_roundings_are_small():
    rounded, x0, _ = _make(True)
    exact, _, _ = _make(False)
    a, b = rounded.grad(0, x0[0], 0), exact.grad(0, x0[0], 0)
    assert 0 < np.linalg.norm(a - b) <= 2.0 ** -6 * np.linalg.norm(b)
