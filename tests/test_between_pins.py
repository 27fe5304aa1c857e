"""Pins of oracle.between: the generator's published test vectors, closed forms, and gradients
against differences."""
import numpy as np
import pytest

from oracle import between


@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_philox_published_vectors(counter, key, want):
    assert tuple(between.philox(counter, key)) == want


def test_mask_share_and_independence():
    keep, factor = between.keep_mask(40, 101, 0.25, 7, 3)
    # 4040 draws: five standard deviations of the share are 0.034
    assert abs(keep.mean() - 0.75) < 0.035 and factor == 4 / 3
    other, _ = between.keep_mask(40, 101, 0.25, 7, 4)
    assert (keep != other).mean() > 0.3
    assert between.keep_mask(3, 9, 0.0, 1, 1)[0].all()
    assert not between.keep_mask(3, 9, 1.0, 1, 1)[0].any()


def _case(seed=3, lengths=(3, 0, 1, 5), d=4):
    rng = np.random.default_rng(seed)
    off = np.concatenate([[0], np.cumsum(lengths)])
    n = int(off[-1])
    x, g, dy = (rng.standard_normal((n, d)) for _ in range(3))
    h0, dlast = (rng.standard_normal((len(lengths), d)) for _ in range(2))
    return x, g, off, dy, h0, dlast


def test_closed_forms():
    x, g, off, _, h0, _ = _case()
    y, last, *_ = between.recur(x, np.full_like(g, 80.0), off, h0)
    np.testing.assert_allclose(last, h0, rtol=1e-12)       # the gate is open: nothing comes in
    y, *_ = between.recur(x, np.full_like(g, -80.0), off, h0)
    np.testing.assert_allclose(y, x, rtol=1e-12)           # it is shut: nothing stays
    # a constant gate: a geometric sum
    n, f = 6, 1 / (1 + np.exp(-0.3))
    ones = np.ones((n, 1))
    y, *_ = between.recur(ones, 0.3 * ones, [0, n])
    np.testing.assert_allclose(y[:, 0], 1 - f ** np.arange(1, n + 1), rtol=1e-14)


def test_gradients_against_differences():
    x, g, off, dy, h0, dlast = _case()

    def loss(x, g, h0):
        y, last, *_ = between.recur(x, g, off, h0)
        return (y * dy).sum() + (last * dlast).sum()

    got, _ = between.recur_grad(x, g, off, dy, h0, dlast)
    step = 1e-5
    for k, (v, grad) in enumerate(zip((x, g, h0), got)):
        for at in np.ndindex(v.shape):
            args = [x, g, h0]
            hi, lo = v.copy(), v.copy()
            hi[at] += step
            lo[at] -= step
            args[k] = hi
            up = loss(*args)
            args[k] = lo
            # second differences: step^2 = 1e-10, and 1e-16 / step of rounding
            assert abs((up - loss(*args)) / (2 * step) - grad[at]) < 1e-8, (k, at)


def test_a_planted_mistake_is_seen():
    """The gradient of the gate with the new state in place of the one before."""
    x, g, off, dy, h0, dlast = _case()
    (dx, dg, _), _ = between.recur_grad(x, g, off, dy, h0, dlast)
    y, _, _, _, before = between.recur(x, g, off, h0)
    wrong = dg * (y - x) / (before - x)
    assert np.abs(wrong - dg).max() > 0.05
