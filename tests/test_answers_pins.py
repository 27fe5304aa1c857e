"""Pins of oracle.answers: the 8-bit type's table, brute-force nearest codes, closed forms and
frequencies of the choice of a token, planted mistakes."""
import numpy as np
import pytest

from oracle import answers


def test_table():
    t = answers.e4m3_table()
    assert t[0] == 0 and t[1] == 2.0 ** -9 and t[7] == 7 * 2.0 ** -9 and t[8] == 2.0 ** -6
    assert t[0x38] == 1 and t[0x7E] == 448 and np.isnan(t[0x7F]) and t[0xB8] == -1
    assert (np.diff(t[:127]) > 0).all()


def test_quantize_by_brute_force():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((6, 300)) * np.exp2(rng.integers(-30, 30, (6, 1)))
    x[2] = 0
    x[3, 7] = 448 * 2.0 ** 40
    codes, scales = answers.quantize(x)
    v, t = answers.values(codes, scales), answers.e4m3_table()
    t = t[~np.isnan(t)]
    assert (v[:, 300:] == 0).all() and (scales[2] == 0).all()
    for i in range(6):
        for b in range(3):
            part = x[i, 128 * b:128 * (b + 1)]
            s = 2.0 ** (float(scales[i, b]) - 127)
            big = np.abs(part).max()
            assert big <= 448 * s and (scales[i, b] == 0 or big > 448 * s / 2)
            have = v[i, 128 * b:128 * b + len(part)]
            best = np.abs(t[:, None] * s - part).min(axis=0)
            np.testing.assert_array_equal(np.abs(have - part), best)
    assert v[3, 7] == 448 * 2.0 ** 40


def test_ties_go_to_the_even_code():
    x = np.array([[448.0, 1 + 1 / 16, 1 + 3 / 16, 2.0 ** -10, 3 * 2.0 ** -10]])
    codes, scales = answers.quantize(x)
    assert scales[0, 0] == 127
    assert answers.values(codes, scales)[0, :5].tolist() == [448, 1, 1.25, 0, 2 * 2.0 ** -9]


def test_sample_closed_forms():
    x = [1.0, 3.0, 2.0, 3.0, -np.inf, np.nan]
    e = np.exp(np.array([-2.0, 0, -1, 0]))
    assert answers.sample(x, 0.999, temperature=0) == (1, 1.0)
    assert answers.sample(x, 0.999, top_k=1) == (1, 1.0)
    assert answers.sample(x, 0.999, top_k=2) == (3, 0.5)
    assert answers.sample(x, 0.4999, top_k=2) == (1, 0.5)
    assert answers.sample(x, 0.5, top_k=2) == (3, 0.5)
    assert answers.sample(x, 0.0)[0] == 0
    assert answers.sample(x, 0.0)[1] == pytest.approx(e[0] / e.sum(), rel=1e-15)
    assert answers.sample(x, 0.0, min_p=0.2)[0] == 1     # exp(-2) is out, exp(-1) is in
    assert answers.sample(x, 0.5, min_p=0.2)[0] == 2
    # the first has 0.40 of the weight, the first two 0.80
    assert answers.sample(x, 0.99, top_p=0.39)[0] == 1
    assert answers.sample(x, 0.99, top_p=0.41)[0] == 3
    assert answers.sample(x, 0.0, top_p=0.0) == (1, 1.0)
    assert answers.sample([np.inf, 1.0, np.inf], 0.6) == (2, 0.5)
    for bad in (dict(u=1.0), dict(u=-0.1), dict(u=np.nan), dict(u=0.5, temperature=-1),
                dict(u=0.5, temperature=np.inf), dict(u=0.5, top_p=np.nan)):
        assert answers.sample(x, **bad) == (-1, 0.0)
    assert answers.sample([-np.inf, np.nan], 0.5) == (-1, 0.0)


def test_sample_frequencies():
    """Over evenly spread random numbers each token comes as often as its probability says."""
    rng = np.random.default_rng(2)
    x = rng.standard_normal(12)
    n = 4000
    got = [answers.sample(x, (i + 0.5) / n, temperature=0.7, top_k=9, top_p=0.9)[0]
           for i in range(n)]
    order = np.argsort(-x)[:9]
    w = np.exp(x[order] / 0.7)
    have = int(np.searchsorted(np.cumsum(w) / w.sum(), 0.9)) + 1
    p = np.zeros(12)
    p[order[:have]] = w[:have] / w[:have].sum()
    assert np.abs(np.bincount(got, minlength=12) / n - p).max() <= 1.5 / n


def test_a_planted_mistake_is_seen():
    """top-p over the weights of all entries instead of those that top-k leaves."""
    x = np.log([4.0, 3.0, 2.0, 1.0, 1.0, 1.0])
    right = answers.sample(x, 0.9, top_k=3, top_p=0.7)[0]   # 4/9, 7/9: two are kept
    wrong = answers.sample(x, 0.9, top_k=3, top_p=0.7 * 12 / 9)[0]
    assert right == 1 and wrong == 2
