"""fp64 CPU oracle of the 4-bit key/value cache: the values that it holds, the
attention over them with the keys' weights, and the choice of slots to keep.

TEST INFRASTRUCTURE ONLY, like the rest of this package; it shares no code with
the HIP kernels or their host library.

A value is a number of the grid 0, 0.5, 1, 1.5, 2, 3, 4, 6 (codes 0 to 7) or its
negative, times a scale: 2^e for 32 channels of a row of K, e the smallest
integer >= -100 with max|x| < 7 * 2^e, but at most 125; s for a row of V, the smallest number of
six significant bits with s >= max|x| / 6 and s >= 2^-100, but at most 21 * 2^121 (6 s stays
a bf16 number). x goes to the nearest
value, ties to the even code. K's 32 channels, or V's row, with a value that
is not finite are NaN.
"""
from __future__ import annotations

import numpy as np

__all__ = ["GRID", "cache_k", "cache_v", "cache_attention", "cache_keep"]

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _nearest(x: np.ndarray, scale: np.ndarray) -> np.ndarray:
    """The value nearest to x. x and the values have few bits: the distances
    are exact in fp64."""
    dist = np.abs(np.abs(x)[..., None] - GRID * scale[..., None])
    best = dist.min(axis=-1, keepdims=True)
    tie = dist == best
    # of two codes at the same distance the even one
    code = np.where(tie, np.where(np.arange(8) % 2 == 0, 0, 1), 2).argmin(axis=-1)
    return np.copysign(GRID[code] * scale, x) + 0.0


def cache_k(k: np.ndarray) -> np.ndarray:
    """The values of rows of K [..., d], d a multiple of 32."""
    x = np.asarray(k, dtype=np.float64)
    x = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    ok = np.isfinite(x).all(axis=-1)
    x = np.where(ok[..., None], x, 0.0)
    m, p = np.frexp(np.abs(x).max(axis=-1))      # max = m 2^p, 0.5 <= m < 1; 7/8 2^(e + 3)
    e = np.maximum(np.where(m > 0, np.minimum(p - 3 + (m >= 0.875), 125), -100), -100)
    y = _nearest(x, np.broadcast_to(np.ldexp(1.0, e)[..., None], x.shape))
    return np.where(ok[..., None], y, np.nan).reshape(np.shape(k))


def cache_v(v: np.ndarray) -> np.ndarray:
    """The values of rows of V [..., d]."""
    x = np.asarray(v, dtype=np.float64)
    ok = np.isfinite(x).all(axis=-1, keepdims=True)
    x = np.where(ok, x, 0.0)
    m, p = np.frexp(np.maximum(np.abs(x).max(axis=-1, keepdims=True) / 6.0, 2.0 ** -100))
    s = np.minimum(np.ldexp(np.ceil(m * 64.0), p - 6), 21 * 2.0 ** 121)
    return np.where(ok, _nearest(x, np.broadcast_to(s, x.shape)), np.nan)


def cache_attention(q, k, v, length: int, count: int, causal: bool, scale: float):
    """One key/value head: q [G, Lq, d], k and v [capacity, d] (the cache's values).
    Returns O [G, Lq, d], A = sum_k P |v_k| [G, Lq, d], pred [G, Lq] and the weights
    [capacity] (P summed over the rows of finite output)."""
    G, Lq, d = q.shape
    o, a = np.zeros((G, Lq, d)), np.zeros((G, Lq, d))
    pred, w = np.zeros((G, Lq)), np.zeros(len(k))
    for i in range(min(count, Lq)):
        n = min(length, length - count + i + 1) if causal else length
        if n <= 0:
            continue
        s = scale * (q[:, i] @ k[:n].T)
        with np.errstate(invalid="ignore"):
            p = np.exp(s - s.max(axis=-1, keepdims=True))
            p /= p.sum(axis=-1, keepdims=True)
            o[:, i], a[:, i] = p @ v[:n], p @ np.abs(v[:n])
            pred[:, i] = p @ v[:n].sum(axis=-1)
        fine = np.isfinite(o[:, i]).all(axis=-1)
        w[:n] += p[fine].sum(axis=0)
    return o, a, pred, w


def cache_keep(w: np.ndarray, length: int, keep: int, recent: int) -> np.ndarray:
    """The slots that one head keeps, in order. NaN counts as larger than all."""
    if length <= keep:
        return np.arange(length)
    old = length - min(recent, keep)
    key = np.where(np.isnan(w[:old]), np.inf, w[:old])
    nan = np.isnan(w[:old])
    # by NaN, then weight (both descending), then slot
    order = np.lexsort((np.arange(old), -key, ~nan))
    return np.concatenate([np.sort(order[:keep - (length - old)]), np.arange(old, length)])
