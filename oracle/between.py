"""What stands between the input layer and the output layer, plainly, in fp64.

TEST INFRASTRUCTURE ONLY (see the package docstring).

  philox     Philox4x32-10 (Salmon, Moraes, Dror and Shaw 2011), in Python integers.
  keep_mask  the mask that lst_dropout documents.
  recur      h_t = f_t h_{t-1} + (1 - f_t) x_t with f = sigmoid(g), over packed sequences.
  recur_grad its gradients, by the chain rule from the last row to the first.

recur and recur_grad also return how far a float32 evaluation may be off, in any order of
association: with u = 2^-24, a gate (exp, one sum, one reciprocal, one product) and its product
and sum are each computed to at most C = 10 roundings, so that the error E_t of a state is at most
f_t E_{t-1} + C u (f_t M_{t-1} + (1 - f_t) |x_t|), with M the same recurrence on absolute values.

Pins: tests/test_between_pins.py (the generator's published test vectors, closed forms of the
recurrence, gradients against differences, planted mistakes).
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24
C = 10


def philox(counter, key):
    """Four 32-bit words of the block with the given counter (4 words) and key (2 words)."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def keep_mask(rows: int, cols: int, p: float, seed: int, offset: int):
    """(rows x cols truth values, the factor of a kept element)."""
    drop = int(p * 65536 + 0.5)
    keep = np.zeros((rows, cols), dtype=bool)
    key = (seed & 0xFFFFFFFF, seed >> 32)
    for i in range(rows):
        for j in range(cols):
            if j % 8 == 0:
                words = philox((j // 8, i, offset & 0xFFFFFFFF, offset >> 32), key)
            keep[i, j] = (words[j % 8 // 2] >> (16 * (j % 2)) & 0xFFFF) >= drop
    return keep, (65536 / (65536 - drop) if drop < 65536 else 0.0)


def _gates(g):
    g = np.asarray(g, dtype=np.float64)
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-g)), 1 / (1 + np.exp(g))


def recur(x, g, offsets, h0=None):
    """(y, h_last, error of y, error of h_last, state before each row)."""
    x = np.asarray(x, dtype=np.float64)
    f, i = _gates(g)
    n = len(offsets) - 1
    last = np.zeros((n, x.shape[1])) if h0 is None else np.array(h0, dtype=np.float64)
    y, before = np.full_like(x, np.nan), np.full_like(x, np.nan)
    err_y, err_last = np.zeros_like(x), np.zeros_like(last)
    for s in range(n):
        h, m, e = last[s], np.abs(last[s]), np.zeros(x.shape[1])
        for t in range(offsets[s], offsets[s + 1]):
            before[t] = h
            e = f[t] * e + C * U * (f[t] * m + i[t] * np.abs(x[t]))
            m = f[t] * m + i[t] * np.abs(x[t])
            h = f[t] * h + i[t] * x[t]
            y[t], err_y[t] = h, e
        last[s], err_last[s] = h, e
    return y, last, err_y, err_last, before


def recur_grad(x, g, offsets, grad_y, h0=None, grad_last=None):
    """(grad_x, grad_g, grad_h0) and the error of each."""
    x, dy = np.asarray(x, dtype=np.float64), np.asarray(grad_y, dtype=np.float64)
    f, i = _gates(g)
    _, last, err_h, _, before = recur(x, g, offsets, h0)
    n = len(offsets) - 1
    dh = np.zeros_like(last) if grad_last is None else np.array(grad_last, dtype=np.float64)
    dx, dg = np.full_like(x, np.nan), np.full_like(x, np.nan)
    err_x, err_g, err_0 = np.zeros_like(x), np.zeros_like(x), np.zeros_like(dh)
    for s in range(n):
        m, size, e = dh[s], np.abs(dh[s]), np.zeros(x.shape[1])
        for t in range(offsets[s + 1] - 1, offsets[s] - 1, -1):
            L, size, e = dy[t] + m, np.abs(dy[t]) + size, e + U * (np.abs(dy[t]) + size)
            dx[t], err_x[t] = i[t] * L, i[t] * (e + C * U * size)
            w, h = f[t] * i[t], before[t]
            dg[t] = (h - x[t]) * w * L
            e_h = err_h[t - 1] if t > offsets[s] else 0.0
            err_g[t] = w * ((e_h + 2 * C * U * (np.abs(h) + np.abs(x[t]))) * size +
                            np.abs(h - x[t]) * e)
            m, e, size = f[t] * L, f[t] * (e + C * U * size), f[t] * size
        dh[s], err_0[s] = m, e
    return (dx, dg, dh), (err_x, err_g, err_0)
