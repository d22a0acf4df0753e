"""Plain 64-bit forms of the norms and of the key/value cache calls, written from their definitions (include/symb_block.h): numpy, segment by segment."""
import numpy as np


def norm_fwd(off, X, weights, biases, layer, eps, base):
    """X [T][d] float64, weights / biases per segment (None as in the C ABI); Y [T][d]."""
    Y = np.empty_like(X)
    for i in range(len(off) - 1):
        x = X[off[i]:off[i + 1]]
        z, _, w = _standard(x, weights[i], layer, eps, base)
        Y[off[i]:off[i + 1]] = z * w + (0.0 if biases[i] is None else biases[i])
    return Y


def _standard(x, weight, layer, eps, base):
    mu = x.mean(1, keepdims=True) if layer else 0.0
    with np.errstate(divide="ignore", invalid="ignore"):
        r = 1.0 / np.sqrt(((x - mu) ** 2).mean(1, keepdims=True) + eps)
        return (x - mu) * r, r, np.ones(x.shape[1]) if weight is None else base + weight


def norm_bwd(off, X, dY, weights, layer, eps, base):
    """(dX, [dweight of every segment], [dbias])"""
    dX, dw, db = np.empty_like(X), [], []
    for i in range(len(off) - 1):
        rows = slice(off[i], off[i + 1])
        z, r, w = _standard(X[rows], weights[i], layer, eps, base)
        g = dY[rows] * w
        dx = g - z * (g * z).mean(1, keepdims=True)
        if layer:
            dx = dx - g.mean(1, keepdims=True)
        dX[rows] = r * dx
        dw.append((dY[rows] * z).sum(0))
        db.append(dY[rows].sum(0))
    return dX, dw, db


def e4m3_values():
    """The 256 values that a byte stands for."""
    b = np.arange(256)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e > 0, (1 + m / 8.0) * 2.0 ** (e - 7.0), m / 8.0 * 2.0 ** -6)
    v[(b & 127) == 127] = np.nan
    return np.where(b < 128, v, -v)


_POSITIVE = e4m3_values()[:127]


def e4m3(x):
    """Nearest value (ties to the even byte) of |x| <= 448; others and NaN become NaN."""
    a = np.abs(x)
    ok = a <= 448                                       # (False for NaN)
    hi = np.searchsorted(_POSITIVE, np.where(ok, a, 0.0))
    hi = np.minimum(hi, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _POSITIVE[hi] - np.where(ok, a, 0.0), np.where(ok, a, 0.0) - _POSITIVE[lo]
    pick = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return np.where(ok, np.copysign(_POSITIVE[pick], x), np.nan)


def turn(x, table, positions, dim, adjacent):
    """x [T][heads][D]: pairs of the first `dim` elements turned by the rows' positions."""
    x = x.copy()
    for t, s in enumerate(positions):
        c, n = table[s, :dim // 2], table[s, dim // 2:dim]
        a, b = (np.arange(0, dim, 2), np.arange(1, dim, 2)) if adjacent else (np.arange(dim // 2), np.arange(dim // 2, dim))
        u, w = x[t][:, a].copy(), x[t][:, b].copy()
        x[t][:, a], x[t][:, b] = u * c - w * n, w * c + u * n
    return x


def append_exact(rows, first, old, old_scale):
    """One page and head: rows [n][D] behind `first` kept tokens `old` [first][D] (real values).  Returns (scale, kept tokens held again, new ones before rounding)."""
    a = np.abs(rows[np.isfinite(rows)])
    top = a.max() if a.size else 0.0
    e = -126
    while top > 448 * 2.0 ** e:
        e += 1
    s = max(2.0 ** e, old_scale) if first else 2.0 ** e
    return s, e4m3(old / s) * s, rows / s


def attention(off, past, K, V, q, scale, window, cap):
    """K, V: per segment [tokens][kv_heads][D] (all of past + new tokens); q [T][heads][D].  Rows see position - window < s <= position.
    Returns (out, sum of |weight x value|, largest |q_d k_d| a row meets): what the error bounds are made of."""
    T, heads, D = q.shape
    out, mass, big = np.zeros(q.shape), np.zeros(q.shape), np.zeros((T, heads, 1))
    for i in range(len(past)):
        for j in range(off[i + 1] - off[i]):
            pos = past[i] + j
            lo = max(0, pos + 1 - window) if window else 0
            t = off[i] + j
            for h in range(heads):
                k, v = K[i][lo:pos + 1, h * K[i].shape[1] // heads], V[i][lo:pos + 1, h * V[i].shape[1] // heads]
                x = scale * (k @ q[t, h])
                if cap:
                    x = cap * np.tanh(x / cap)
                w = np.exp(x - x.max()) if not np.isnan(x).any() else np.full(len(x), np.nan)
                w = w / w.sum()
                out[t, h], mass[t, h] = w @ v, w @ np.abs(v)
                big[t, h, 0] = np.abs(k * q[t, h]).max() * scale
    return out, mass, big
