"""Pins of oracle.answers' 4-bit values and log probabilities: brute-force nearest values, closed
forms, differences, planted mistakes."""
import numpy as np
import pytest

from oracle import answers


def test_quantize_four_by_brute_force():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((6, 75)) * np.exp2(rng.integers(-30, 30, (6, 1)))
    x[2] = 0
    x[3, 7] = 6 * 2.0 ** 40
    codes, scales = answers.quantize_four(x)
    v = answers.values_four(codes, scales)
    assert codes.shape == (6, 48) and scales.shape == (6, 3)
    assert (v[:, 75:] == 0).all() and (scales[2] == 0).all()
    t = np.concatenate([answers.E2M1, -answers.E2M1])
    for i in range(6):
        for b in range(3):
            part = x[i, 32 * b:32 * (b + 1)]
            s = 2.0 ** (float(scales[i, b]) - 127)
            big = np.abs(part).max()
            assert big <= 6 * s and (scales[i, b] == 0 or big > 6 * s / 2)
            have = v[i, 32 * b:32 * b + len(part)]
            np.testing.assert_array_equal(np.abs(have - part),
                                          np.abs(t[:, None] * s - part).min(axis=0))
    assert v[3, 7] == 6 * 2.0 ** 40


def test_four_bit_ties_signs_and_what_is_not_finite():
    x = np.array([[6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -5, -0.0]])
    codes, scales = answers.quantize_four(x)
    assert scales.tolist() == [[127]]
    assert answers.values_four(codes, scales)[0, :11].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, 0, -4, 0]
    assert codes[0, 4] & 15 == 8 and codes[0, 5] & 15 == 8  # the sign of a zero
    codes, scales = answers.quantize_four(np.array([[1.0] * 32 + [np.inf] + [1.0] * 31]))
    assert scales.tolist() == [[125, 255]] and codes[0, 16] & 15 == 0
    assert np.isnan(answers.values_four(codes, scales)[0, 32:]).all()


def test_logprobs_closed_forms():
    x = [1.0, 3.0, 2.0, 3.0, -np.inf, np.nan]
    e = np.exp(np.array([-2.0, 0, -1, 0]))
    logp, h, ids, best = answers.logprobs(x, [0, 3, 4, -1, 6], top=5)
    np.testing.assert_allclose(logp, [-2 - np.log(e.sum()), -np.log(e.sum()), -np.inf, 0, 0])
    p = e / e.sum()
    assert h == pytest.approx(-(p * np.log(p)).sum(), rel=1e-14)
    assert ids.tolist() == [1, 3, 2, 0, -1] and best[4] == -np.inf
    assert best[1] == logp[1]
    # twice the temperature is half of the row
    a, b = answers.logprobs(x, [2], 2.0), answers.logprobs(np.array(x) / 2, [2])
    assert a[0] == pytest.approx(b[0]) and a[1] == pytest.approx(b[1])
    assert answers.logprobs([0.0] * 8, [5])[1] == pytest.approx(np.log(8))
    assert answers.logprobs([np.inf, 1.0, np.inf], [0, 1])[0].tolist() == [-np.log(2), -np.inf]
    for bad in (0.0, -1.0, np.inf, np.nan):
        assert answers.logprobs([1.0, 2.0], [0], bad, 1)[0][0] == -np.inf
    logp, h, ids, _ = answers.logprobs([-np.inf] * 3, [1, -1], top=2)
    assert logp.tolist() == [-np.inf, 0] and h == 0 and ids.tolist() == [-1, -1]


def test_logprobs_gradient_against_differences():
    rng = np.random.default_rng(3)
    x = rng.standard_normal(11)
    x[4] = -np.inf
    tokens, g, ge, t = [2, 2, 9, -1, 4], rng.standard_normal(5), 0.7, 1.3
    alive = x > -np.inf

    def total(x):
        logp, h, _, _ = answers.logprobs(x, tokens, t)
        return (np.where(np.isfinite(logp), logp, 0) * g)[:4].sum() + ge * h

    grad = answers.logprobs_grad(x, tokens, g, ge, t)
    assert grad[4] == 0 and grad.sum() == pytest.approx(0, abs=1e-14)
    for _ in range(5):
        u = np.where(alive, rng.standard_normal(11), 0)
        y = np.where(alive, x, 0)
        step = lambda s: total(np.where(alive, y + s * u, -np.inf))  # noqa: E731
        assert (step(1e-6) - step(-1e-6)) / 2e-6 == pytest.approx((grad * u).sum(), rel=1e-6,
                                                                  abs=1e-8)
    # a mistake: a token named twice that counted once
    assert np.abs(grad - answers.logprobs_grad(x, tokens[1:], g[1:], ge, t)).max() > 1e-3
