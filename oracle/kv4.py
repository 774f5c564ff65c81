"""The 4-bit cache format in 64 bits (test-only): microscaled groups of 32.

A group of 32 consecutive dims of one token and KV head stands for
code * 2^e: codes are E2M1 values (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their
negatives), e the smallest exponent with max|x| <= 7 * 2^e, within
[-127, 125].  7 lies half a step past the largest code (the step below 6 is
2), so no value is off by more than half the step around it.  Values round to
the nearest code, of two as near to the one with the even code; a group with
an infinity or a NaN is NaN throughout.
"""
from __future__ import annotations

import numpy as np

from .gemv import bf16_to_f32

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
E_MIN, E_MAX = -127, 125


def exponents(x: np.ndarray) -> np.ndarray:
    """e of every group; x [..., 32] finite, fp64."""
    top = np.abs(x).max(-1)
    e = np.full(top.shape, E_MIN)
    for i in np.ndindex(top.shape):
        c = E_MIN
        while top[i] > 7.0 * 2.0 ** c and c < E_MAX:
            c += 1
        e[i] = c
    return e


def exponents_fast(x: np.ndarray) -> np.ndarray:
    """The same in closed form: top / 2^e in (3.5, 7]."""
    top = np.abs(x).max(-1)
    m, ex = np.frexp(top)  # top = m 2^ex, m in [1/2, 1)
    e = ex - 3 + (m > 0.875)
    return np.where(top == 0, E_MIN, np.clip(e, E_MIN, E_MAX))


def round_to_grid(a: np.ndarray) -> np.ndarray:
    """Nearest grid value of a >= 0, ties to the even code, saturating."""
    lo = np.clip(np.searchsorted(GRID, a, side="right") - 1, 0, 6)
    mid = (GRID[lo] + GRID[lo + 1]) / 2
    up = (a > mid) | ((a == mid) & (lo % 2 == 1))
    return GRID[np.where(up, lo + 1, lo)]


def stored(u16: np.ndarray) -> np.ndarray:
    """What bf16 values [..., D] (raw bits, D a multiple of 32) read back as
    from a 4-bit pool, in fp64."""
    x = bf16_to_f32(u16).astype(np.float64)
    g = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    bad = ~np.isfinite(g).all(-1, keepdims=True)
    g = np.where(bad, 0.0, g)
    s = np.ldexp(1.0, exponents_fast(g))[..., None]
    y = np.copysign(round_to_grid(np.abs(g) / s) * s, g)
    return np.where(bad, np.nan, y).reshape(x.shape)


def attend(q, k, v, scale=None):
    """o [G, D] of queries q [G, D] over k, v [L, D], all fp64."""
    if k.shape[0] == 0:
        return np.zeros_like(q)
    s = (q @ k.T) * (1 / np.sqrt(q.shape[1]) if scale is None else scale)
    p = np.exp(s - s.max(1, keepdims=True))
    return (p / p.sum(1, keepdims=True)) @ v
