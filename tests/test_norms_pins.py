"""Pins of oracle.norms: closed forms, differences, planted mistakes."""
import numpy as np
import pytest

from oracle import norms


def test_closed_forms():
    y, q = norms.norm([[3.0, 4.0], [0.0, 0.0]], [1.0, 2.0], 0.0 + 1e-300)
    assert q[0] == pytest.approx(1 / np.sqrt(12.5), rel=1e-15)
    np.testing.assert_allclose(y[0], [3 / np.sqrt(12.5), 8 / np.sqrt(12.5)], rtol=1e-15)
    assert (y[1] == 0).all()
    y, _ = norms.norm(np.full((1, 7), -5.0), np.ones(7), 0.0)
    np.testing.assert_allclose(y, -1, rtol=1e-15)


def test_gradients_against_differences():
    rng = np.random.default_rng(0)
    s, gy, gs = (rng.standard_normal((5, 9)) for _ in range(3))
    w, eps, h = rng.standard_normal(9), 0.1, 1e-6
    total = lambda s, w: (norms.norm(s, w, eps)[0] * gy).sum() + (s * gs).sum()  # noqa: E731
    ds, dw = norms.norm_grad(s, w, eps, gy, gs)
    for _ in range(5):
        u, v = rng.standard_normal(s.shape), rng.standard_normal(9)
        assert (total(s + h * u, w) - total(s - h * u, w)) / (2 * h) == pytest.approx(
            (ds * u).sum(), rel=1e-7, abs=1e-7)
        assert (total(s, w + h * v) - total(s, w - h * v)) / (2 * h) == pytest.approx(
            (dw * v).sum(), rel=1e-7, abs=1e-7)
    # a mistake: without the mean's term the gradient is another one
    q = norms.norm(s, w, eps)[1]
    assert np.abs(ds - (q[:, None] * gy * w + gs)).max() > 1e-3


def test_clip():
    n, f, out = norms.clip([[3.0], [[0.0, 4.0]]], 1.0)
    assert n == 5 and f == 0.2 and out[1][0, 1] == pytest.approx(0.8)
    assert norms.clip([[3.0, 4.0]], 5.0)[1] == 1.0
    assert norms.clip([[3.0, np.inf]], 5.0)[1] == 1.0
    assert np.isnan(norms.clip([[3.0, np.nan]], 5.0)[0])
    assert norms.clip([], 1.0)[:2] == (0.0, 1.0)
