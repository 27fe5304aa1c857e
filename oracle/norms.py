"""Root-mean-square norm of rows with its gradients, and gradient clipping, plainly, in fp64.

TEST INFRASTRUCTURE ONLY (see the package docstring).

  norm       y = s w / sqrt(mean(s^2) + eps) of rows s, and each row's factor.
  norm_grad  gradients with respect to s and w.
  clip       the norm over all gradients, and the gradients scaled to a largest one.

Pins: tests/test_norms_pins.py (closed forms, differences, planted mistakes).
"""
from __future__ import annotations

import math

import numpy as np


def norm(s, w, eps):
    """(y, q): q the factor of each row."""
    s, w = np.asarray(s, dtype=np.float64), np.asarray(w, dtype=np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        q = 1.0 / np.sqrt((s * s).sum(axis=1) / s.shape[1] + eps)
        return s * q[:, None] * w, q


def norm_grad(s, w, eps, grad_y, grad_sum=None):
    """(dL/ds, dL/dw) for dL/dy = grad_y and what else of dL/ds there is."""
    _, q = norm(s, w, eps)
    s, grad_y = np.asarray(s, dtype=np.float64), np.asarray(grad_y, dtype=np.float64)
    hat = s * q[:, None]
    a = grad_y * w
    ds = q[:, None] * (a - hat * (a * hat).mean(axis=1, keepdims=True))
    if grad_sum is not None:
        ds = ds + grad_sum
    return ds, (grad_y * hat).sum(axis=0)


def clip(tensors, max_norm):
    """(norm, factor, scaled tensors); nothing is scaled where the norm is not finite."""
    total = math.fsum(float(v) ** 2 for t in tensors for v in np.asarray(t, np.float64).ravel())
    n = math.sqrt(total) if not math.isnan(total) else total
    factor = max_norm / n if math.isfinite(n) and n > max_norm else 1.0
    return n, factor, [np.asarray(t, dtype=np.float64) * factor for t in tensors]
