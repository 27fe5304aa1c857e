"""What follows the output layer, plainly, in fp64.

TEST INFRASTRUCTURE ONLY (see the package docstring).

  quantize  rows in e4m3 with one power-of-two scale for each block of 128 columns.
  values    what codes and scales stand for.
  scores    O = H W^T of quantised rows, and how far float32 sums may be off.
  sample    the token that lst_sample chooses.
  quantize_four, values_four  the same in e2m1, one scale for each block of 32 columns.
  logprobs  log probabilities of given tokens, the entropy and the likeliest tokens.
  logprobs_grad  the gradient of a weighted sum of the first two.

Pins: tests/test_answers_pins.py and tests/test_probabilities_pins.py (the type's value table, brute-force nearest codes, closed forms
and frequencies of the choice, differences of the logarithms, planted mistakes).
"""
from __future__ import annotations

import numpy as np

BLOCK = 128
U = 2.0 ** -24


def e4m3_table():
    """Value of each of the 256 codes: sign, 4 bits of exponent (bias 7), 3 bits; 127 is no number."""
    v = np.zeros(256)
    for c in range(256):
        e, f = c >> 3 & 15, c & 7
        v[c] = (8 + f) * 2.0 ** (e - 10) if e else f * 2.0 ** -9
        if c & 127 == 127:
            v[c] = np.nan
        if c & 128:
            v[c] = -v[c]
    return v


_UP = e4m3_table()[:127]


def _nearest(a):
    """Code of each magnitude (at most 448), to nearest, ties to the even code."""
    hi = np.searchsorted(_UP, a).clip(max=126)
    lo = np.maximum(hi - 1, 0)
    up, down = _UP[hi] - a, a - _UP[lo]
    return np.where((up < down) | ((up == down) & (hi % 2 == 0)) | (a == _UP[hi]), hi, lo)


def quantize(x):
    """(codes, scales) as bytes: rows of whole blocks, biased exponents."""
    x = np.asarray(x, dtype=np.float64)
    n, d = x.shape
    b = -(-d // BLOCK)
    pad = np.zeros((n, b * BLOCK))
    pad[:, :d] = x
    pad = pad.reshape(n, b, BLOCK)
    fine = np.isfinite(pad)
    size = np.where(fine, np.abs(pad), 0.0)
    big = size.max(axis=2)
    e = np.full(big.shape, -127)
    for at in np.ndindex(big.shape):
        if big[at] > 0:
            k = int(np.frexp(big[at])[1]) - 10
            while 448 * 2.0 ** k < big[at]:
                k += 1
            e[at] = max(k, -127)
    codes = _nearest(size / 2.0 ** e[:, :, None].astype(float))
    codes = np.where(fine, codes | np.where(np.signbit(pad), 128, 0), 127)
    return codes.reshape(n, b * BLOCK).astype(np.uint8), (e + 127).astype(np.uint8)


def values(codes, scales):
    s = 2.0 ** (np.asarray(scales, dtype=float) - 127)
    return e4m3_table()[codes] * np.repeat(s, BLOCK, axis=1)


def scores(H, W):
    """(H W^T, its bar): a float32 sum in any order, of terms that are exact, may be off by one
    step (two halves, should the unit cut instead of round) for each of its terms."""
    O = H @ W.T
    return O, 2 * U * (H.shape[1] + 2) * (np.abs(H) @ np.abs(W).T)


def sample(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, its probability among those kept) from one row of outputs: -1 for none."""
    x = np.asarray(x, dtype=np.float64)
    u, t, p, q = (float(np.float32(v)) for v in (u, temperature, top_p, min_p))
    if not (0 <= u < 1 and 0 <= t < np.inf) or np.isnan(p) or np.isnan(q):
        return -1, 0.0
    alive = np.flatnonzero(~np.isnan(x) & (x > -np.inf))
    if not len(alive):
        return -1, 0.0
    order = alive[np.argsort(-x[alive], kind="stable")]
    top = x[order[0]]
    if t == 0:
        return int(order[0]), 1.0
    if top_k > 0:
        order = order[:top_k]
    # entries as large as the largest weigh 1, also where that is infinite
    w = np.array([1.0 if v == top else float(np.exp((v - top) / t)) for v in x[order]])
    kept = 0
    total, run = w.sum(), 0.0
    for v in w:
        if kept and (v < q or (p < 1 and not run < p * total)):
            break
        run += v
        kept += 1
    by = np.argsort(order[:kept])
    sums = np.cumsum(w[by])
    j = int(np.searchsorted(sums, u * sums[-1], side="right"))
    return int(order[by[j]]), w[by[j]] / sums[-1]


SMALL = 32
E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def quantize_four(x):
    """(codes, scales) as bytes: two codes a byte, the lower column in the lower half; biased
    exponents, 255 for a block with a value that is not finite."""
    x = np.asarray(x, dtype=np.float64)
    n, d = x.shape
    b = -(-d // SMALL)
    pad = np.zeros((n, b * SMALL))
    pad[:, :d] = x
    pad = pad.reshape(n, b, SMALL)
    fine = np.isfinite(pad)
    size = np.where(fine, np.abs(pad), 0.0)
    big = size.max(axis=2)
    e = np.full(big.shape, -127)
    for at in np.ndindex(big.shape):
        if big[at] > 0:
            k = int(np.frexp(big[at])[1]) - 4
            while 6 * 2.0 ** k < big[at]:
                k += 1
            e[at] = max(k, -127)
    a = size / 2.0 ** e[:, :, None].astype(float)
    hi = np.searchsorted(E2M1, a).clip(max=7)
    lo = np.maximum(hi - 1, 0)
    up, down = E2M1[hi] - a, a - E2M1[lo]
    codes = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    codes = codes | np.where(fine & np.signbit(pad), 8, 0)
    codes = codes.reshape(n, b * SMALL // 2, 2)
    scales = np.where(fine.all(axis=2), e + 127, 255)
    return (codes[:, :, 0] | codes[:, :, 1] << 4).astype(np.uint8), scales.astype(np.uint8)


def values_four(codes, scales):
    c = np.asarray(codes)
    c = np.stack((c & 15, c >> 4), axis=2).reshape(c.shape[0], -1)
    s = np.where(np.asarray(scales) == 255, np.nan, 2.0 ** (np.asarray(scales, dtype=float) - 127))
    return np.where(c > 7, -E2M1[c & 7], E2M1[c & 7]) * np.repeat(s, SMALL, axis=1)


def _weights(x, temperature):
    """(z, weights relative to the largest, which entries have any) of one row; None for a row
    without an entry, or with a temperature that is not above zero and finite."""
    x = np.asarray(x, dtype=np.float64)
    t = float(np.float32(temperature))
    alive = ~np.isnan(x) & (x > -np.inf)
    if not alive.any() or not 0 < t < np.inf:
        return None
    top = x[alive].max()
    if top == np.inf:  # the infinite ones alone, all alike
        alive = alive & (x == top)
        z = np.where(alive, 0.0, -np.inf)
    else:
        z = np.where(alive, (np.where(alive, x, top) - top) / t, -np.inf)
    return z, np.where(alive, np.exp(z), 0.0), alive


def logprobs(x, tokens, temperature=1.0, top=0):
    """(log probability of each token, entropy, ids and log probabilities of the `top` likeliest)
    of one row.  A token of -1, or outside the row, is unused: 0."""
    x = np.asarray(x, dtype=np.float64)
    D = len(x)
    used = [0 <= t < D for t in tokens]
    none = np.full(top, -1, dtype=int), np.full(top, -np.inf)
    got = _weights(x, temperature)
    if got is None:
        return np.array([-np.inf if u else 0.0 for u in used]), 0.0, *none
    z, w, alive = got
    # entries whose weight is too small for a float keep their logarithm
    log = np.where(alive, z - np.log(w.sum()), -np.inf)
    p = w / w.sum()
    entropy = -(p * np.where(w > 0, log, 0.0)).sum()
    order = np.flatnonzero(alive)
    order = order[np.argsort(-x[order], kind="stable")][:top]
    ids, best = none
    ids[:len(order)], best[:len(order)] = order, log[order]
    return np.array([log[t] if u else 0.0 for t, u in zip(tokens, used)]), entropy, ids, best


def logprobs_grad(x, tokens, grad_logp, grad_entropy=0.0, temperature=1.0):
    """Gradient of sum_k grad_logp[k] logp_k + grad_entropy entropy with respect to the row."""
    x = np.asarray(x, dtype=np.float64)
    got = _weights(x, temperature)
    if got is None:
        return np.zeros_like(x)
    z, w, alive = got
    logp, entropy, _, _ = logprobs(x, tokens, temperature)
    p = w / w.sum()
    log = np.where(w > 0, z - np.log(w.sum()), 0.0)
    grad = -p * grad_entropy * (log + entropy)
    for t, g, lp in zip(tokens, grad_logp, logp):
        if 0 <= t < len(x) and np.isfinite(lp):
            grad = grad - g * p
            grad[t] += g
    return grad / float(np.float32(temperature))
