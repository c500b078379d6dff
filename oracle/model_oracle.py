"""Plain fp64 definitions of the operators around a model's linear layers (test infrastructure only).

Written from the formulas, with NumPy, and independent of the CUDA library: layer
norm with and without a mean, embedding lookups, and the Muon step.
"""
from __future__ import annotations

import numpy as np


# ------------------------------------------------------------------ norms

def norm(x, w, b, layer, eps):
    """(y, mean, rstd) of fp64 rows x [R, d]; w and b may be None."""
    mean = x.mean(1) if layer else np.zeros(len(x))
    c = x - mean[:, None]
    rstd = 1 / np.sqrt((c * c).mean(1) + eps)
    y = c * rstd[:, None]
    if w is not None:
        y = y * w
    return (y if b is None else y + b), mean, rstd


def norm_backward(x, w, layer, mean, rstd, dy):
    """(dx, dw, db) for given statistics."""
    n = (x - mean[:, None] if layer else x) * rstd[:, None]
    h = dy if w is None else dy * w
    dx = h - n * (h * n).mean(1, keepdims=True)
    if layer:
        dx = dx - h.mean(1, keepdims=True)
    return dx * rstd[:, None], (dy * n).sum(0), dy.sum(0)
