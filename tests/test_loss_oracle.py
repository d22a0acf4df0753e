"""oracle/loss.py against the definitions worked row by row, and its gradients against differences.  No GPU needed."""
import math

import numpy as np
import pytest

from oracle import loss as ol


def _case(seed, cap):
    rng = np.random.default_rng(seed)
    off = np.array([0, 2, 2, 7])
    X, W = rng.standard_normal((7, 8)) * 2, rng.standard_normal((11, 8))
    labels = np.array([3, -1, 10, 0, -100, 5, 5])
    ids = np.array([[1, 2, 3], [-1, -1, -1], [4, -2, 4], [9, 8, -1], [0, 0, 0], [10, 1, 5], [7, 6, 2]])
    return rng, off, X, W, labels, ids, rng.standard_normal((7, 3)) * 2, [0.5, 9.0, 2.0], [2.0, 1.0, 0.7]


def _z(x, w, cap):
    s = float(x @ w)
    return cap * math.tanh(s / cap) if cap else s


@pytest.mark.parametrize("cap", [0.0, 2.5])
@pytest.mark.parametrize("mean", [True, False])
def test_against_the_definition(mean, cap):
    _, off, X, W, labels, ids, logits, scales, temps = _case(1, cap)
    loss, L = ol.cross_entropy(off, X, W, labels, scales, mean, cap)[:2]
    for t, y in enumerate(labels):
        z = [_z(X[t], w, cap) for w in W]
        assert L[t] == pytest.approx(0 if y < 0 else -math.log(math.exp(z[y]) / sum(map(math.exp, z))), rel=1e-12)
    assert loss == pytest.approx([L[0], 0, L[2:].sum() / (4 if mean else 1)])
    loss, L = ol.distillation(off, X, W, ids, logits, scales, temps, mean, cap)[:2]
    for t in range(7):
        T = temps[0] if t < 2 else temps[2]
        z, mine = [_z(X[t], w, cap) / T for w in W], [j for j in range(3) if ids[t, j] >= 0]
        q = [math.exp(logits[t, j] / T) for j in mine]
        kl = sum(a / sum(q) * (math.log(a / sum(q)) - math.log(math.exp(z[ids[t, j]]) / sum(map(math.exp, z)))) for a, j in zip(q, mine))
        assert L[t] == pytest.approx(T * T * kl, rel=1e-12)
    assert loss == pytest.approx([L[0], 0, L[2:].sum() / (5 if mean else 1)])


@pytest.mark.parametrize("cap", [0.0, 2.5])
@pytest.mark.parametrize("teacher", [False, True])
def test_gradients_against_differences(teacher, cap):
    rng, off, X, W, labels, ids, logits, scales, temps = _case(2, cap)
    f = (lambda x: ol.distillation(off, x, W, ids, logits, scales, temps, True, cap)) if teacher else (lambda x: ol.cross_entropy(off, x, W, labels, scales, True, cap))
    dX, mass = f(X)[2:4]
    assert (np.abs(dX) <= mass + 1e-15).all()
    step = 1e-5
    for t in range(7):
        for k in range(8):
            up, down = X.copy(), X.copy()
            up[t, k] += step
            down[t, k] -= step
            assert dX[t, k] == pytest.approx(np.dot(scales, f(up)[0] - f(down)[0]) / (2 * step), rel=1e-6, abs=1e-8)


def test_rows_far_from_their_label():
    X, W = np.array([[900.0], [900.0]]), np.array([[-1.0], [1.0], [0.0]])
    _, L, dX = ol.cross_entropy([0, 2], X, W, np.array([0, 1]), [1.0], False)[:3]
    assert L == pytest.approx([1800.0, 0.0]) and dX[0] == pytest.approx(2.0) and dX[1] == pytest.approx(0.0)
