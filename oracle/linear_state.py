"""Linear attention with a decay for each head, token by token in float64, and rotary positions (test infrastructure).

Beside each result stand the sums of its terms' magnitudes, which the rounding bounds of the tests go by.
"""
from __future__ import annotations

import numpy as np

from .paged_cache import to_bf16  # noqa: F401


def attend(Q, K, V, decay, S0, scale):
    """One sequence: Q [T, Hq, D], K, V [T, Hkv, D], decay g [T, Hkv], S0 [Hkv, D, D].  Returns o, S, and the magnitudes: of
    o's terms, of S's, and what fp32 roundings of S at every token (two of 2^-24 each) come to at the end."""
    T, Hq, D = Q.shape
    H = K.shape[1]
    q = Q.astype(np.float64).reshape(T, H, Hq // H, D)
    k, v = K.astype(np.float64), V.astype(np.float64)
    keep = np.exp(decay.astype(np.float64))
    S = S0.astype(np.float64).copy()
    A, E = np.abs(S), np.zeros_like(S)
    o, oa = np.zeros((T, H, Hq // H, D)), np.zeros((T, H, Hq // H, D))
    with np.errstate(invalid="ignore", over="ignore"):
        for t in range(T):
            g = keep[t][:, None, None]
            S = g * S + k[t][:, :, None] * v[t][:, None, :]
            A = g * A + np.abs(k[t])[:, :, None] * np.abs(v[t])[:, None, :]
            E = g * E + 2.0 ** -23 * A
            o[t] = scale * (q[t] @ S)
            oa[t] = scale * (np.abs(q[t]) @ A)
    return o.reshape(T, Hq, D), S, oa.reshape(T, Hq, D), A, E


def frequencies(pairs, base=10000.0, scaling="none", factor=1.0, original=0, slow=1.0, fast=32.0):
    """Radians a position of each pair, axis by axis, and the magnitude of cos and sin."""
    out = []
    for p in pairs:
        for i in range(p):
            b = base * factor ** (p / (p - 1.0)) if scaling == "base" else base
            f = b ** (-i / p)
            if scaling == "linear":
                f /= factor
            elif scaling == "ramp":
                w = min(1.0, max(0.0, (original * f / (2 * np.pi) - slow) / (fast - slow)))
                f = (1.0 - w) * f / factor + w * f
            out.append(f)
    return out, 0.1 * np.log(factor) + 1.0 if scaling == "ramp" else 1.0


def angles(positions, pairs, freq):
    """positions [T, axes] (whole numbers) -> angles [T, sum(pairs)] modulo a turn, in extended precision."""
    axis = np.repeat(np.arange(len(pairs)), pairs)
    turn = 2 * np.longdouble("3.14159265358979323846264338327950288")
    a = positions[:, axis].astype(np.longdouble) * np.array(freq, np.longdouble)[None, :]
    return np.fmod(a, turn).astype(np.float64)


def rotate(X, angle, magnitude, style):
    """X [T, heads, D], angle [T, R / 2]: the first R channels of each head turned, in float64."""
    R = 2 * angle.shape[1]
    y = X.astype(np.float64).copy()
    c, s = magnitude * np.cos(angle)[:, None, :], magnitude * np.sin(angle)[:, None, :]
    i, j = (slice(0, R // 2), slice(R // 2, R)) if style == "half" else (slice(0, R, 2), slice(1, R, 2))
    a, b = y[..., i].copy(), y[..., j].copy()
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    return y
