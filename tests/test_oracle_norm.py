"""Pins of the RMS norm's oracle: direct values and central differences."""

import numpy as np
import pytest

from oracle import norm as orc


def test_forward_by_hand():
    s = np.array([[3.0, 4.0], [0.0, -2.0]])
    y = orc.forward(s, [1.0, 0.5], 0.0)
    r0, r1 = 1 / np.sqrt(12.5), 1 / np.sqrt(2.0)
    assert np.allclose(y, [[3 * r0, 2 * r0], [0.0, -r1]], rtol=1e-15)
    assert np.allclose(orc.forward(np.zeros((1, 4)), np.ones(4), 1e-6), 0.0)
    assert orc.scales(np.array([[1.0, -448.0, 0.0, 2.0, 896.0]]), 2).tolist() == [
        [1.0, 2.0 / 448.0, 2.0]]
    assert orc.scales(np.zeros((1, 3)), 0).tolist() == [[2.0 ** -126]]


@pytest.mark.parametrize("H,eps", [(1, 1e-3), (2, 0.0), (7, 1e-6), (33, 0.1)])
def test_backward_is_the_derivative(H, eps):
    rng = np.random.default_rng(H)
    s, w, dy = rng.normal(size=(3, H)), rng.normal(size=H), rng.normal(size=(3, H))
    extra = rng.normal(size=(3, H))
    dx, dw, _, _ = orc.backward(dy, s, w, eps, extra)

    def loss(s, w):
        return (orc.forward(s, w, eps) * dy).sum() + (s * extra).sum()
    h = 1e-6
    for i in np.ndindex(*s.shape):
        d = np.zeros_like(s)
        d[i] = h
        assert abs((loss(s + d, w) - loss(s - d, w)) / (2 * h) - dx[i]) < 1e-7 * (1 + abs(dx[i]))
    for i in range(H):
        d = np.zeros(H)
        d[i] = h
        assert abs((loss(s, w + d) - loss(s, w - d)) / (2 * h) - dw[i]) < 1e-7 * (1 + abs(dw[i]))
