"""Losses through a vocabulary matrix in 64 bits, from the formulas of include/symb_loss.h: numpy arrays in, numpy arrays out."""
import numpy as np


def _rows(X, W, cap):
    s = X.astype(np.float64) @ W.astype(np.float64).T
    if not cap:
        return s, np.ones_like(s)
    e = np.exp(-2 * np.minimum(np.abs(s / cap), 350))      # (1 - tanh^2 would cancel)
    return cap * np.tanh(s / cap), 4 * e / (1 + e) ** 2


def _softmax(z):
    e = np.exp(z - z.max(1, keepdims=True))
    return e / e.sum(1, keepdims=True)


def _finish(off, part, L, D, P, slope, W, scales, mean):
    """Losses of the segments, of the rows, the gradient; for bounds, the magnitudes of the terms with p - q added up, and of those with p + q."""
    loss, (dX, mass, both) = np.zeros(len(off) - 1), np.zeros((3, len(part), W.shape[1]))
    for i in range(len(off) - 1):
        rows = slice(off[i], off[i + 1])
        n = max(part[rows].sum(), 1) if mean else 1
        loss[i] = L[rows].sum() / n
        dX[rows] = (D[rows] * slope[rows]) @ W * (scales[i] / n)
        mass[rows] = np.abs(D[rows] * slope[rows]) @ np.abs(W) * abs(scales[i] / n)
        both[rows] = (P[rows] * slope[rows]) @ np.abs(W) * abs(scales[i] / n)
    dX[~part] = mass[~part] = both[~part] = 0
    return loss, L, dX, mass, both


def cross_entropy(off, X, W, labels, scales, mean=True, cap=0.0):
    """labels negative: the row takes no part."""
    part = labels >= 0
    X = np.where(part[:, None], X, 0)
    z, slope = _rows(X, W, cap)
    t = np.arange(len(labels))
    own = z[t, labels * part]
    rest = np.exp(np.minimum(z - own[:, None], 700))
    rest[t, labels * part] = 0
    far = z.max(1) - own > 600                     # (beyond what exp holds the others are all there is)
    top = z.max(1)
    L = np.where(far, top - own + np.log(np.exp(z - top[:, None]).sum(1)), np.log1p(rest.sum(1)))
    D = _softmax(z)
    P = D.copy()
    P[t, labels * part] += 1
    D[t, labels * part] = -np.where(far, 1.0, rest.sum(1) / (1 + rest.sum(1)))
    D[~part] = 0
    return _finish(off, part, np.where(part, L, 0.0), D, P, slope, W.astype(np.float64), scales, mean)


def distillation(off, X, W, ids, logits, scales, temperatures, mean=True, cap=0.0):
    """ids negative: no entry."""
    there = ids >= 0
    part = there.any(1)
    X = np.where(part[:, None], X, 0)
    T = np.repeat(np.asarray(temperatures, np.float64), np.diff(off))[:, None]
    z, slope = _rows(X, W, cap)
    z = z / T
    l = np.where(there, logits.astype(np.float64) / T, -np.inf)
    l[~part] = 0
    q = np.where(there, _softmax(l), 0.0)
    logp = z - z.max(1, keepdims=True)
    logp -= np.log(np.exp(logp).sum(1, keepdims=True))
    mine = np.take_along_axis(logp, np.where(there, ids, 0), 1)
    L = T[:, 0] ** 2 * np.where(q > 0, q * (np.log(np.where(q > 0, q, 1.0)) - mine), 0.0).sum(1)
    D, P, at = np.exp(logp), np.exp(logp), (np.arange(len(ids))[:, None], np.where(there, ids, 0))
    np.add.at(D, at, -q)
    np.add.at(P, at, q)
    D[~part] = 0
    return _finish(off, part, np.where(part, L, 0.0), D * T, P * T, slope, W.astype(np.float64), scales, mean)
