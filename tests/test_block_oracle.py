"""Pins of the plain forms in oracle/block.py: gradients against central differences, the 8-bit rounding against its definition, attention against a weighted mean."""
import numpy as np
import pytest
import torch

from oracle import block as ob


@pytest.mark.parametrize("layer", [True, False])
def test_norm_gradients_are_the_differences_of_the_forward(layer):
    rng = np.random.default_rng(1)
    off, d = [0, 3, 3, 5], 7
    X, dY = rng.standard_normal((5, d)) + 0.5, rng.standard_normal((5, d))
    w = [rng.standard_normal(d), None, rng.standard_normal(d)]
    b = [rng.standard_normal(d), None, None]
    dX, dw, db = ob.norm_bwd(off, X, dY, w, layer, 1e-5, 1.0)
    loss = lambda X, w, b: (dY * ob.norm_fwd(off, X, w, b, layer, 1e-5, 1.0)).sum()  # noqa: E731
    h = 1e-5
    for t in range(5):
        for k in range(d):
            p, m = X.copy(), X.copy()
            p[t, k] += h
            m[t, k] -= h
            assert abs((loss(p, w, b) - loss(m, w, b)) / (2 * h) - dX[t, k]) < 1e-7
    for i in (0, 2):
        for k in range(d):
            e = np.zeros(d)
            e[k] = h
            up, down = [x if j != i else x + e for j, x in enumerate(w)], [x if j != i else x - e for j, x in enumerate(w)]
            assert abs((loss(X, up, b) - loss(X, down, b)) / (2 * h) - dw[i][k]) < 1e-7
    up, down = [b[0] + h, None, None], [b[0] - h, None, None]
    assert abs((loss(X, w, up) - loss(X, w, down)) / (2 * h) - db[0].sum()) < 1e-7
    assert not dw[1].any() and not db[1].any()


def test_e4m3_values_and_rounding():
    bytes_ = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    v = ob.e4m3_values()
    np.testing.assert_array_equal(v, bytes_)
    assert v[0x7e] == 448 and v[1] == 2.0 ** -9 and np.isnan(v[0x7f]) and np.isnan(v[0xff])
    x = np.concatenate([np.random.default_rng(2).uniform(-448, 448, 20000), np.random.default_rng(3).uniform(-0.03, 0.03, 20000), v[~np.isnan(v)],
                        (v[:126] + v[1:127]) / 2])
    got = ob.e4m3(x)
    d = np.abs(x[:, None] - v[None, ~np.isnan(v)]).min(1)
    np.testing.assert_allclose(np.abs(got - x), d, atol=1e-12)
    ties = (v[:126] + v[1:127]) / 2
    byte = np.searchsorted(v[:127], ob.e4m3(ties))
    assert (byte % 2 == 0).all()
    assert np.isnan(ob.e4m3(np.array([np.inf, -np.inf, np.nan, 500.0]))).all()


def test_page_scale_is_the_smallest_power_of_two_that_fits():
    for top, want in ((448.0, 1.0), (448.1, 2.0), (224.0, 0.5), (3.5, 2.0 ** -7), (1e-3, 2.0 ** -18), (0.0, 2.0 ** -126)):
        s, _, new = ob.append_exact(np.array([[top, -top / 3]]), 0, np.zeros((0, 2)), 0.0)
        assert s == want and np.abs(new).max() <= 448
    s, kept, _ = ob.append_exact(np.array([[900.0, np.inf]]), 1, np.array([[3.0, -1.25]]), 0.5)
    assert s == 4.0 and kept.tolist() == [[3.0, -1.25]]                     # a power of two: held again as they were


def test_attention_is_a_weighted_mean():
    rng = np.random.default_rng(4)
    K, V, q = [rng.standard_normal((9, 2, 4))], [rng.standard_normal((9, 2, 4))], rng.standard_normal((3, 4, 4))
    out, mass, _ = ob.attention([0, 3], [6], K, V, q, 0.5, 0, 0.0)
    x = 0.5 * np.einsum("d,sd->s", q[1, 3], K[0][:8, 1])
    w = np.exp(x) / np.exp(x).sum()
    np.testing.assert_allclose(out[1, 3], np.einsum("s,sd->d", w, V[0][:8, 1]), rtol=1e-12)
    assert (mass >= np.abs(out) - 1e-12).all()
    one, _, _ = ob.attention([0, 3], [6], K, V, q, 0.5, 1, 0.0)            # a window of one token: its own value
    np.testing.assert_allclose(one[2, 0], V[0][8, 0], rtol=1e-12)
    soft, _, _ = ob.attention([0, 3], [6], K, V, q, 0.5, 0, 1e6)           # a large cap changes nothing
    np.testing.assert_allclose(soft, out, rtol=1e-6)
