"""Plain CPU statement of the paged 8-bit cache: rotation, held values, masked attention (test infrastructure).

Rotation is done in fp32 with every product and sum rounded by itself, as the cache defines it, so held values
can be compared bit for bit; attention is done in fp64 from the held values.
"""
from __future__ import annotations

import numpy as np

__all__ = ["rotate", "held", "attention", "to_bf16"]


def to_bf16(x: np.ndarray) -> np.ndarray:
    """fp32 -> the nearest bf16 value (ties to even), as fp32; finite inputs."""
    b = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    b = (b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000
    return b.astype(np.uint32).view(np.float32).reshape(x.shape)


def rotate(x: np.ndarray, cos: np.ndarray, sin: np.ndarray, style: str) -> np.ndarray:
    """x [tokens][heads][D] fp32, cos / sin [tokens][R / 2] fp32 -> rotated, fp32."""
    x = x.astype(np.float32)
    R = 2 * cos.shape[1]
    y = x.copy()
    c, s = cos[:, None, :], sin[:, None, :]
    if style == "half":
        i, j = slice(0, R // 2), slice(R // 2, R)
    else:
        i, j = slice(0, R, 2), slice(1, R, 2)
    a, b = x[..., i], x[..., j]
    y[..., i] = (a * c).astype(np.float32) - (b * s).astype(np.float32)
    y[..., j] = (b * c).astype(np.float32) + (a * s).astype(np.float32)
    return y


def _e4m3(x: np.ndarray) -> np.ndarray:
    """Nearest E4M3 value (ties to even, saturating at 448) of fp64 values."""
    a = np.abs(x)
    with np.errstate(divide="ignore"):
        e = np.floor(np.log2(np.where(a > 0, a, 1.0)))
    step = np.exp2(np.maximum(e, -6) - 3)
    return np.clip(np.rint(x / step) * step, -448, 448)


def held(x: np.ndarray, page: int) -> np.ndarray:
    """x [tokens][heads][D] (one sequence from its first token on) as the cache holds it, fp64."""
    out = np.zeros(x.shape, dtype=np.float64)
    for p in range(0, len(x), page):
        for h in range(x.shape[1]):
            b = x[p: p + page, h].astype(np.float64)
            top = np.max(np.where(np.isfinite(b), np.abs(b), 0.0))
            e = -120
            while top > 448 * 2.0 ** e:
                e += 1
            b = np.where(np.isnan(b), 0.0, b)
            b = np.where(np.isinf(b), np.sign(b) * 448 * 2.0 ** e, b)
            out[p: p + page, h] = _e4m3(b * 2.0 ** -e) * 2.0 ** e
    return out


def attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, causal: bool, window: int, sinks: int, scale=None):
    """q [n_q][Hq][D], k / v [n][Hkv][D] -> fp64 [n_q][Hq][D]; query i stands at n - n_q + i."""
    nq, Hq, D = q.shape
    n, Hkv = k.shape[:2]
    G = Hq // Hkv
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    p = (n - nq + np.arange(nq))[:, None]
    j = np.arange(n)[None, :]
    see = np.broadcast_to(j <= p, (nq, n)) if causal else np.ones((nq, n), bool)
    if window > 0:
        see = see & ((j > p - window) | (j < sinks))
    out = np.zeros((nq, Hq, D))
    for h in range(Hq):
        s = (q[:, h].astype(np.float64) @ k[:, h // G].astype(np.float64).T) * scale
        s = np.where(see, s, -np.inf)
        m = np.max(s, axis=1, keepdims=True, initial=-1e300)
        w = np.exp(s - m)
        t = w.sum(1, keepdims=True)
        out[:, h] = np.where(t > 0, w @ v[:, h // G].astype(np.float64) / np.where(t > 0, t, 1.0), 0.0)
    return out
