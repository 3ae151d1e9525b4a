"""The head of a training step in numpy, fp64: layer norm, dropout and softmax cross entropy with their gradients,
written from their definitions, row by row where the definition is."""
from __future__ import annotations

import numpy as np

MASK = (1 << 64) - 1
GOLDEN = 0x9E3779B97F4A7C15


def mix64(z: int) -> int:
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & MASK
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & MASK
    return z ^ (z >> 31)


def kept(n: int, p: float, seed: int, first: int) -> np.ndarray:
    """[n] of truth values: which elements of a call dropout keeps.  p is rounded to fp32."""
    key, limit = mix64(seed & MASK), int(float(np.float32(p)) * 2.0 ** 32)
    out = np.empty(n + 1, dtype=bool)
    for w in range((n + 1) // 2):
        word = mix64((key + (first + w) * GOLDEN) & MASK)
        out[2 * w], out[2 * w + 1] = (word & 0xFFFFFFFF) >= limit, (word >> 32) >= limit
    return out[:n]


def dropout(x, p, seed, first):
    keep = kept(x.size, p, seed, first).reshape(x.shape)
    scale = 0.0 if p >= 1.0 else 1.0 / (1.0 - float(np.float32(p)))
    return np.where(keep, x.astype(np.float64) * scale, 0.0)


def layernorm(x, gamma, beta, eps):
    x = x.astype(np.float64)
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    return (x - mean[:, None]) * rstd[:, None] * gamma + beta, mean, rstd


def layernorm_backward(x, gamma, gy, eps):
    """dx, dgamma, dbeta of sum <gy, layernorm(x)>."""
    x, gy = x.astype(np.float64), gy.astype(np.float64)
    _, mean, rstd = layernorm(x, gamma, 0.0, eps)
    xhat = (x - mean[:, None]) * rstd[:, None]
    a = gy * gamma
    dx = rstd[:, None] * (a - a.mean(1, keepdims=True) - xhat * (a * xhat).mean(1, keepdims=True))
    return dx, (gy * xhat).sum(0), gy.sum(0)


def softmax_xent(h, V, b, label):
    """loss, lse [N]; rows with label -1 are 0, rows whose label names no class NaN."""
    h, V = h.astype(np.float64), V.astype(np.float64)
    loss, lse = np.zeros(len(label)), np.zeros(len(label))
    for n, c in enumerate(label):
        if c == -1:
            continue
        z = V @ h[n] + (0.0 if b is None else b)
        top = z.max()
        lse[n] = top + np.log(np.exp(z - top).sum())
        loss[n] = lse[n] - z[c] if 0 <= c < len(V) else np.nan
    return loss, lse


def softmax_xent_backward(h, V, b, label, gloss):
    """dh, dV, db of sum <gloss, loss>, and what their rounding errors are measured by: the derivatives of the logits
    g [N, C] and the softmax p [N, C]."""
    h, V = h.astype(np.float64), V.astype(np.float64)
    N, C = len(label), len(V)
    g, p = np.zeros((N, C)), np.zeros((N, C))
    for n, c in enumerate(label):
        if c == -1:
            continue
        z = V @ h[n] + (0.0 if b is None else b)
        e = np.exp(z - z.max())
        p[n] = e / e.sum()
        g[n] = p[n] * gloss[n] if 0 <= c < C else np.nan
        if 0 <= c < C:
            g[n, c] -= gloss[n]
    used = np.asarray(label) != -1
    return g @ V, g[used].T @ h[used], g.sum(0), g, p
