"""Plain fp64 definitions of the training-side operators (test infrastructure only).

Written from the formulas, with NumPy, and independent of the CUDA library:
token log-probabilities under a softmax, the clipped policy loss with a KL
term, the preference loss over pairs, AdamW with 32- and 8-bit moments, and
the factored second moments of a matrix.
"""
from __future__ import annotations

import numpy as np

MASK64 = (1 << 64) - 1


# ------------------------------------------------------------------ log-probabilities

def token_logprobs(x, targets, tau):
    """(logp, lse, entropy) of fp64 logits x [R, V]."""
    x = np.asarray(x, np.float64)
    out = np.zeros((3, x.shape[0]))
    for r, t in enumerate(targets):
        if t < 0:
            continue
        z = x[r] / tau
        if np.all(z == -np.inf):
            out[:, r] = -np.inf, -np.inf, 0.0
            continue
        top = z.max()
        if not top < np.inf:                     # +inf, or NaN
            out[:, r] = np.nan
            continue
        e = np.exp(z - top)
        s = e.sum()
        p = e / s
        logq = z - top - np.log(s)               # exact where top is of any size
        out[:, r] = logq[t], top + np.log(s), -(p * np.where(p > 0, logq, 0.0)).sum()
    return out


def token_logprobs_backward(x, targets, tau, w, h):
    """d (sum w logp + sum h entropy) / dx."""
    x = np.asarray(x, np.float64)
    d = np.zeros_like(x)
    logp, lse, ent = token_logprobs(x, targets, tau)
    for r, t in enumerate(targets):
        if t < 0 or lse[r] == -np.inf or (w[r] == 0 and h[r] == 0):
            continue
        q = x[r] / tau - lse[r]
        p = np.exp(q)
        d[r] = -w[r] * p - h[r] * p * (np.where(p > 0, q, 0.0) + ent[r])
        d[r, t] += w[r]
    return d / tau


# ------------------------------------------------------------------ losses

def policy_loss(logp, old, ref, ent, adv, mask, low, high, kl_coef, ent_coef, reduction, norm):
    """A dict of the loss, its parts, statistics and gradients; mask is boolean [B, T]."""
    B, T = logp.shape
    z = np.zeros((B, T))
    lp, lo = np.where(mask, logp, 0.0), np.where(mask, old, 0.0)
    a = np.broadcast_to(adv[:, None] if adv.ndim == 1 else adv, (B, T))
    a = np.where(mask, a, 0.0)
    ratio = np.exp(lp - lo)
    free, held = ratio * a, np.clip(ratio, 1 - low, 1 + high) * a
    clip = free > held
    l = -np.minimum(free, held)
    grad = np.where(clip, 0.0, -free)
    k = z
    if ref is not None:
        gap = np.where(mask, ref, 0.0) - lp
        k = np.expm1(gap) - gap
    if kl_coef:
        l = l + kl_coef * k
        grad = grad - kl_coef * np.expm1(gap)
    if ent_coef:
        l = l - ent_coef * np.where(mask, ent, 0.0)
    n = mask.sum(1).astype(np.float64)
    if reduction == "token_mean":
        w = np.full(B, 1 / max(n.sum(), 1.0))
    elif reduction == "seq_mean":
        w = 1 / (B * np.maximum(n, 1.0))
    else:
        w = np.full(B, 1 / (B * norm))
    seq = (l * mask).sum(1) * w
    total = max(n.sum(), 1.0)
    return dict(loss=seq.sum(), seq=seq, w=w,
                stats=np.array([(k * mask).sum() / total, (clip & mask).sum() / total, n.sum()]),
                d=grad * mask * w[:, None], dh=-ent_coef * mask * w[:, None])


def preference_loss(logp, ref, mask, kind, beta, margin, eps, mean):
    P = logp.shape[0] // 2
    gap = np.where(mask, logp, 0.0) - (0.0 if ref is None else np.where(mask, ref, 0.0))
    n = np.maximum(mask.sum(1), 1).astype(np.float64) if mean else np.ones(2 * P)
    s = gap.sum(1) / n
    x = beta * (s[:P] - s[P:]) - margin

    def f(y):
        if kind == "sigmoid":
            return np.logaddexp(0.0, -y), -np.exp(-np.logaddexp(0.0, y))
        if kind == "hinge":
            return np.maximum(0.0, 1 - y), np.where(y < 1, -1.0, 0.0)
        return ((y - 0.5) / beta) ** 2, 2 * (y - 0.5) / beta ** 2
    (a, da), (b, db) = f(x), f(-x)
    pair = (1 - eps) * a + eps * b
    slope = ((1 - eps) * da - eps * db) * beta / max(P, 1)
    d = np.concatenate([slope, -slope]) / n
    return dict(loss=pair.mean() if P else 0.0, pair=pair, rewards=beta * s,
                d=d[:, None] * mask)


# ------------------------------------------------------------------ AdamW

def adamw(p, g, m, v, lr, b1, b2, eps, step, wd):
    """(p, m, v) after a step, in fp64 (m, v not rounded)."""
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    up = m / (1 - b1 ** step) / (np.sqrt(v / (1 - b2 ** step)) + eps)
    return p - lr * (up + wd * p), m, v


def mix64(x: int) -> int:
    """The SplitMix64 finaliser."""
    x &= MASK64
    x = ((x ^ (x >> 30)) * 0xBF58476D1CE4E5B9) & MASK64
    x = ((x ^ (x >> 27)) * 0x94D049BB133111EB) & MASK64
    return x ^ (x >> 31)


def chance(n, seed, step, tensor):
    """The 16 random bits of each of a tensor's n elements."""
    key = mix64(tensor ^ mix64(seed ^ mix64(step)))
    out = np.zeros(-(-n // 4) * 4, np.int64)
    for q in range(-(-n // 4)):
        h = mix64(key + (q + 1) * 0x9E3779B97F4A7C15)
        out[4 * q:4 * q + 4] = [(h >> s) & 0xFFFF for s in (0, 16, 32, 48)]
    return out[:n]


def code_values(second: bool):
    """The value of every code: positive ones 2^e (1 + f / 8), code 0 is zero."""
    bits = 8 if second else 7
    k = np.arange(1 << bits)
    y = 2.0 ** (k // 8 - (31 if second else 15)) * (1 + (k % 8) / 8)
    y[0] = 0.0
    return y if second else np.concatenate([y, -y])


def quantise(x, second, rnd):
    """(codes, fp32 scales) of fp32 values x: with y = |x| / scale between two
    codes' values, the upper one is taken if the part of the step above the lower
    one plus rnd / 2^16 reaches 1."""
    x = np.asarray(x, np.float32)
    n = x.size
    levels = np.float32(code_values(second)[:256 if second else 128])
    codes = np.zeros(n, np.int64)
    scales = np.zeros(-(-n // 256), np.float32)
    for b in range(scales.size):
        part = slice(256 * b, min(n, 256 * b + 256))
        a = np.abs(x[part])
        top = a.max()
        if top == 0:
            continue
        scales[b] = max(np.float32(top * np.float32(1 / 1.875)), np.float32(2.0 ** -126))
        y = a * (np.float32(1) / scales[b])
        # as fractions of a binade: the codes' levels are evenly spaced in each
        e = np.floor(np.log2(np.maximum(y.astype(np.float64), 2.0 ** -140)))
        at = (e + (31 if second else 15)) * 8 + (y / 2.0 ** e - 1) * 8
        k = np.floor(at + rnd[part] / 65536.0).astype(np.int64)
        k = np.clip(k, 0, len(levels) - 1)
        if second:
            k = np.where(a > 0, np.maximum(k, 1), 0)
        codes[part] = k
    if not second:
        codes = codes + np.where(x < 0, 128, 0)
    return codes.astype(np.uint8), scales


def dequantise(codes, scales, second):
    return code_values(second)[codes] * np.repeat(scales.astype(np.float64), 256)[:codes.size]


# ------------------------------------------------------------------ factored moments

def factor_moments(v, correction, floor):
    v = np.asarray(v, np.float64) * correction + floor
    return v.mean(1), v.mean(0) / v.mean()
