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


# ------------------------------------------------------------------ embedding

def embedding(table, ids, scale):
    """scale table[id] of fp64 rows; a negative id gives zeros."""
    return np.stack([scale * table[i] if i >= 0 else np.zeros(table.shape[1]) for i in ids])


def embedding_backward(dy, ids, scale, V):
    """(the table's gradient [V, d], the same of magnitudes)."""
    out = np.zeros((2, V, dy.shape[1]))
    for r, i in enumerate(ids):
        if 0 <= i < V:
            out[0, i] += scale * dy[r]
            out[1, i] += abs(scale) * np.abs(dy[r])
    return out[0], out[1]


# ------------------------------------------------------------------ Muon

def newton_schulz(u, coefficients):
    """The iteration on u / |u|_F, short side first."""
    n = np.linalg.norm(u)
    x = u / n if n > 0 else np.zeros_like(u)
    if u.shape[0] > u.shape[1]:
        return newton_schulz(u.T, coefficients).T
    for a, b, c in coefficients:
        g = x @ x.T
        x = a * x + (b * g + c * g @ g) @ x
    return x


def muon_step(w, g, m, lr, beta, nesterov, coefficients, ortho_scale, weight_decay):
    """(w, m, X) after the step, all fp64."""
    m = beta * m + (1 - beta) * g
    u = beta * m + (1 - beta) * g if nesterov else m
    x = newton_schulz(u, coefficients)
    return w - lr * (ortho_scale * x + weight_decay * w), m, x
